"""The calls on a cache in pages against their fp64 reference, through the binding.

Bounds of an attention result (eps = half a step of the type, 2^-24 in fp32, 2^-8 in bf16; A = sum of weights times |v|):
  a logit of D fp32 products and their sum, scaled:  ez = (D + 3) 2^-24 max_j(scale sum |q k|)
  a weight exp2(z - m): the argument's rounding 2 2^-24 |z|, the hardware exponential 2 2^-24, together with both logits'
  errors  ew = 2 ez + 2^-22 (max |z| + 1), |z| <= the bound that ez starts from
  the sums over n rows, in any order and through rescalings and joins: (n + 64) 2^-24 each
  bf16: the weights rounded for the matrix products (eps A), the output rounded (eps |out|).
So |out - exact| <= A (2 ew + 2 (n + 64) 2^-24 + [bf16] 2^-8) + eps |exact|, |lse - exact| <= ew + (n + 64) 2^-24 + 2^-22 |lse|,
each with its products of errors: a factor of 1.02."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_ref as ref
from paper_2507_19906_amd import binding as cd
from tests import helpers as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Setup:
    """Pages in random order, filled; what no query may read holds NaN, entries that no row needs hold rubbish."""

    def __init__(self, lens, nq, hq, hkv, d, dtype, page, window=0, sinks=0, prefix=0, seed=0, spare_tokens=0, one=False, freed=True, scale=0.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.nq, self.hq, self.hkv, self.d, self.page = lens, nq, hq, hkv, d, page
        self.window, self.sinks, self.prefix, self.scale = window, sinks, prefix, scale
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.dt, nb = dt, len(lens)
        need = [-(-n // page) for n in lens]
        first = -(-prefix // page)
        self.max_pages = max(1, max(need)) + 1
        self.n_pages = first + sum(need) + 1
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.k = torch.randn((self.n_pages, hkv, page, d), generator=g).to(dt)
        self.v = torch.randn((self.n_pages, hkv, page, d), generator=g).to(dt)
        self.shared, at, self.table = order[:first], first, []
        for m in need:
            self.table.append(order[at:at + m] + [(1 << 30) if m % 2 else -7] * (self.max_pages - m))
            at += m
        self.offs = np.concatenate([[0], np.cumsum(nq)]).tolist()
        self.total = self.offs[-1] + spare_tokens
        self.q = (torch.randn((self.total, hq, d), generator=g) * 2).to(dt)
        # rows nobody sees: behind the ends, the last page, and under a window everything before the first query's
        seen = torch.zeros((self.n_pages, page), dtype=torch.bool)
        for r in range(prefix):
            seen[self.shared[r // page], r % page] = True
        for b, n in enumerate(lens):
            for r in range(n):
                i0 = n - nq[b]
                if nq[b] and not (window and freed and r <= i0 - window and r >= sinks):
                    seen[self.table[b][r // page], r % page] = True
        hide = ~seen[:, None, :, None].expand(-1, hkv, -1, d)
        self.k[hide], self.v[hide] = NAN, NAN
        if window and freed:                               # freed pages: their entries name nothing any more
            for b, n in enumerate(lens):
                for e in range(need[b]):
                    if not any(seen[self.table[b][e]].tolist()):
                        self.table[b][e] = -5
        self.one = one
        p = cd.make_paged_params(dtype=dt, batch=nb, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=self.n_pages,
                                 max_pages=self.max_pages, window=window, sinks=sinks, scale=scale)
        self.cache = cd.PagedCache(p, self.k.to(DEV), self.v.to(DEV), ints(self.table), ints(lens))
        self.qd = self.q.to(DEV)
        self.out = torch.full((self.total, hq, d), 77.0, dtype=dt, device=DEV)
        self.lse = torch.full((self.total, hq), 77.0, device=DEV)
        self.q_off = None if one else ints(self.offs)
        self.shared_table = ints(self.shared)
        self.most = dict(max_q_len=max(1, max(nq)), max_cache_len=max(lens))
        self.cache.reserve(self.total, self.most["max_q_len"], self.most["max_cache_len"], prefix)
        self.cache.workspace.fill_(255)                     # NaN partials wherever a call reads what it has not written

    def run(self, stream=None):
        if self.prefix:
            self.cache.attend_shared(self.qd, self.out, self.lse, self.shared_table, self.prefix, q_offsets=self.q_off, stream=stream, **self.most)
        else:
            self.cache.attend(self.qd, self.out, self.lse, q_offsets=self.q_off, stream=stream, **self.most)
        return self

    def check(self, sequences=None):
        torch.cuda.synchronize()
        out, lse = self.out.float().cpu().numpy().astype(np.float64), self.lse.cpu().numpy().astype(np.float64)
        kn, vn, qn = (x.float().numpy() for x in (self.k, self.v, self.q))
        eps = 2.0 ** -8 if self.dt == torch.bfloat16 else 2.0 ** -24
        worst = 0.0
        for b in sequences if sequences is not None else range(len(self.lens)):
            lo, hi, n = self.offs[b], self.offs[b + 1], self.lens[b]
            if lo == hi:
                continue

            def rows(pages):
                safe = [e if 0 <= e < self.n_pages else self.n_pages - 1 for e in self.table[b]]
                own = np.concatenate([pages[e].transpose(1, 0, 2) for e in safe])[:n] if n else pages[0].transpose(1, 0, 2)[:0]
                if not self.prefix:
                    return own
                return np.concatenate([np.concatenate([pages[e].transpose(1, 0, 2) for e in self.shared])[:self.prefix], own])
            pos = np.arange(n - (hi - lo), n)
            want = ref.attend(qn[lo:hi], rows(kn), rows(vn), pos, self.scale or self.d ** -0.5, self.window, self.sinks, self.prefix)
            ez = (self.d + 3) * 2.0 ** -24 * want["zabs"]
            ew = 2 * ez + 2.0 ** -22 * (want["zabs"] + 1)
            es = (want["seen"][:, None] + 64) * 2.0 ** -24
            tol = 1.02 * (want["absv"] * (2 * ew + 2 * es + (eps if eps > 1e-5 else 0))[..., None] + eps * np.abs(want["out"])) + 1e-37
            empty = want["seen"] == 0
            assert (out[lo:hi][empty] == 0).all() and (lse[lo:hi][empty] == -np.inf).all()
            err = np.abs(out[lo:hi] - want["out"]) / tol
            assert np.isfinite(out[lo:hi]).all() and err.max() <= 1, (b, err.max(), np.unravel_index(err.argmax(), err.shape))
            some = ~empty
            tl = 1.02 * (ew + es + 2.0 ** -22 * np.abs(np.where(some[:, None], want["lse"], 0)))
            assert (np.abs(lse[lo:hi][some] - want["lse"][some]) <= tl[some]).all(), b
            worst = max(worst, err.max())
        spare = slice(self.offs[-1], self.total)
        assert (out[spare] == 77).all() and (lse[spare] == 77).all()
        return worst


TYPES = [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)]
HEADS = [(8, 2), (4, 4), (3, 1), (16, 1), (10, 2)]


# ---- attention: single tokens ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [1, 5, 16, 32, 48, 64])
def test_one_token(dtype, d, page):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 200, 300, 0]
    Setup(lens, [1] * 16, 8, 2, d, dtype, page, one=True, seed=page).run().check()


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("dtype,d", TYPES)
def test_head_layouts_and_a_few_tokens(hq, hkv, dtype, d):
    # two to six tokens each, more tokens than rows (the first ones see nothing), none at all
    Setup([70, 3, 0, 131, 40], [3, 5, 2, 6, 0], hq, hkv, d, dtype, 16, spare_tokens=2, seed=hq).run().check()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (7, 1), (32, 4), (33, 32), (100, 5), (64, 200), (500, 7), (97, 1), (90, 30), (190, 2), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_one_token_under_a_window(dtype, d, window, sinks):
    lens = [1, 5, 32, 33, 40, 100, 131, 132, 133, 260, 0]
    Setup(lens, [1] * 11, 8, 2, d, dtype, 16, window, sinks, one=True, seed=window % 97).run().check()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_one_token_of_long_caches_split_over_workgroups(dtype, d):
    s = Setup([5000, 1, 129, 0, 2600], [1] * 5, 8, 2, d, dtype, 48, one=True, seed=3).run()
    s.check()
    assert len(H.captured_launches(lambda: s.run())) == 2


@pytest.mark.parametrize("dtype,d", TYPES)
def test_long_window_split_over_workgroups(dtype, d):
    Setup([7000, 600, 4000], [2, 1, 3], 8, 2, d, dtype, 16, 3000, 40, seed=4).run().check()


# ---- attention: prompts and chunks --------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("hq,hkv", HEADS)
def test_prompts(dtype, d, hq, hkv):
    nq = [1, 17, 64, 65, 130, 0, 200]
    Setup(nq, nq, hq, hkv, d, dtype, 16, spare_tokens=3, seed=5).run().check()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [1, 7, 32, 48, 64, 128])
def test_chunks_behind_a_cache(dtype, d, page):
    Setup([300, 129, 77, 64, 50], [40, 129, 33, 10, 60], 6, 2, d, dtype, page, spare_tokens=1, seed=6).run().check()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 2), (31, 0), (64, 4), (65, 70), (128, 33), (1000, 3), (190, 2), (60, 1)])
def test_prompts_and_chunks_under_a_window(dtype, d, window, sinks):
    Setup([300, 129, 400, 64, 50], [300, 129, 60, 10, 60], 6, 2, d, dtype, 16, window, sinks, seed=7).run().check()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_a_chunk_behind_a_long_cache(dtype, d):
    Setup([4000, 1500], [50, 100], 8, 2, d, dtype, 64, seed=8).run().check()


def test_a_longer_prompt():
    Setup([1100, 700], [1100, 513], 4, 1, 128, "bf16", 64, seed=9).run().check()


def test_scale_and_large_logits():
    # weights of one row only, logits of some hundreds: the running maximum moves by more than any exponent
    for dtype in ("bf16", "fp32"):
        Setup([500, 90], [70, 1], 4, 2, 64, dtype, 16, scale=6.0, seed=10).run().check()


# ---- attention behind a shared prefix ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("prefix,page", [(1, 16), (31, 7), (100, 16), (129, 64), (2500, 48)])
def test_shared_prefix_one_token(dtype, d, prefix, page):
    Setup([1, 0, 20, 65, 300, 33], [1] * 6, 8, 2, d, dtype, page, prefix=prefix, one=True, seed=11).run().check()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("hq,hkv", HEADS)
def test_shared_prefix_some_tokens(dtype, d, hq, hkv):
    Setup([4, 0, 20, 65, 90], [4, 2, 0, 30, 70], hq, hkv, d, dtype, 16, prefix=333, spare_tokens=2, seed=12).run().check()


def test_shared_prefix_of_a_large_batch():
    lens = [(7 * b) % 60 for b in range(70)]
    Setup(lens, [1] * 70, 16, 4, 128, "bf16", 16, prefix=1500, one=True, seed=13).run().check(range(0, 70, 9))


def test_the_prefix_equals_one_cache_each():
    s = Setup([3, 60, 9], [3, 2, 1], 8, 2, 128, "bf16", 16, prefix=160, seed=14).run()
    joined = [s.shared + [e for e in row if 0 <= e < s.n_pages] for row in s.table]
    wide = max(map(len, joined))
    p = cd.make_paged_params(dtype="bf16", batch=3, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=s.n_pages, max_pages=wide)
    c = cd.PagedCache(p, s.cache.k_pages, s.cache.v_pages, ints([r + [0] * (wide - len(r)) for r in joined]), ints([163, 220, 169]))
    c.reserve(6, 3, 220)
    out, lse = torch.empty_like(s.out), torch.empty_like(s.lse)
    c.attend(s.qd, out, lse, q_offsets=s.q_off, max_q_len=3, max_cache_len=220)
    torch.cuda.synchronize()
    # both within the bound of the exact result, 2^-8 A + 2^-8 |out| and small terms; A < 4 for normal v (a mean of |v|)
    assert (out.float() - s.out.float()).abs().max() < 2 * (4 + 4) * 2.0 ** -8
    assert (lse - s.lse).abs().max() < 1e-4


@pytest.mark.parametrize("prefix", [0, 70])
@pytest.mark.parametrize("nb,nq,hq,hkv,dtype", [(5000, 1, 2, 1, "bf16"), (4500, 20, 2, 1, "bf16"), (3, 1, 800, 800, "fp32"), (2, 40, 520, 520, "bf16"),
                                                (2, 1, 2000, 125, "bf16")])
def test_many_sequences_and_many_heads(prefix, nb, nq, hq, hkv, dtype):
    # more blocks than are added up on the device, more KV heads than workgroups to share them: a workgroup per block
    lens = [nq + (b * 37) % 50 for b in range(nb)]
    Setup(lens, [nq] * nb, hq, hkv, 64, dtype, 32, prefix=prefix, seed=15).run().check(range(0, nb, max(1, nb // 4)) if hq < 100 else [0])


@pytest.mark.parametrize("dtype,d", TYPES)
def test_both_forms_of_a_call(dtype, d):
    # one launch where every block has a workgroup, two where workgroups share the tiles
    def launches(lens, nq, **kw):
        s = Setup(lens, nq, 8, 2, d, dtype, 32, seed=16, **kw)
        n = len(H.captured_launches(lambda: s.run()))
        s.run().check([0])
        return n
    assert launches([90] * 70, [1] * 70, one=True) == 1 and launches([3000], [1], one=True) == 2
    assert launches([100] * 3, [100] * 3) == 1 and launches([6000], [40]) == 2
    assert launches([50, 3], [1, 1], one=True, prefix=300) == 2


@pytest.mark.parametrize("dtype,d", TYPES)
def test_empty_caches(dtype, d):
    Setup([0, 0, 0], [1, 1, 1], 8, 2, d, dtype, 16, one=True, seed=19).run().check()
    Setup([0, 0, 0], [2, 40, 0], 8, 2, d, dtype, 16, seed=19).run().check()
    Setup([0, 0, 0], [1, 1, 1], 8, 2, d, dtype, 16, prefix=45, one=True, seed=19).run().check()
    Setup([0, 0, 0], [2, 40, 0], 8, 2, d, dtype, 16, prefix=45, seed=19).run().check()


@pytest.mark.parametrize("lens,nq,prefix", [([70, 33], [1, 1], 0), ([4000, 33], [3, 2], 0), ([200, 130], [200, 90], 0), ([6000], [70], 0),
                                            ([30, 70], [20, 1], 500)])
def test_results_in_the_place_of_the_queries(lens, nq, prefix):
    s = Setup(lens, nq, 8, 2, 128, "bf16", 16, prefix=prefix, seed=20)
    s.out = s.qd
    s.run().check()


def test_lengths_that_cannot_be():
    # below zero: no rows; above what the host was told: cut off there, the queries ending at the cut
    s = Setup([40, 70, 90], [2, 1, 3], 8, 2, 64, "bf16", 16, seed=17)
    s.cache.cache_lens.copy_(ints([-5, 70, 1 << 30]))
    s.run()
    torch.cuda.synchronize()
    assert (s.out[:2] == 0).all() and (s.lse[:2] == -math.inf).all()
    s.check([1, 2])                                         # max_cache_len is 90


def test_offsets_that_cannot_be():
    # falling, and beyond the tokens: what is in range is computed, nothing else is touched
    s = Setup([40, 70, 90], [2, 1, 3], 8, 2, 64, "bf16", 16, seed=18, spare_tokens=2)
    s.q_off = ints([0, 2, 1, 1 << 30])
    s.run()
    torch.cuda.synchronize()
    got = s.out[:2].clone()
    s.q_off = ints(s.offs)
    s.run().check()
    assert torch.equal(got[:1], s.out[:1])


@pytest.mark.parametrize("lens,nq,prefix", [([70, 33, 9], [1, 3, 2], 0), ([300, 200, 64], [130, 0, 7], 0), ([4000, 33], [3, 2], 0),
                                            ([30, 70, 12], [20, 1, 12], 333)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_offsets_without_a_bound(dtype, lens, nq, prefix):
    s = Setup(lens, nq, 8, 2, 64, dtype, 16, prefix=prefix, seed=38, spare_tokens=2)
    del s.most["max_q_len"]
    s.cache.reserve(s.total, s.total, max(lens), prefix)
    s.run().check()


@pytest.mark.parametrize("lens,nq,prefix", [([70, 33, 9], [1, 3, 2], 0), ([4000, 300], [30, 2], 0), ([30, 70, 12], [20, 1, 12], 333), ([5, 9], [1, 1], 4000)])
def test_a_bound_far_above_the_tokens(lens, nq, prefix):
    # the largest bound there is (2^26 rows of a KV head): launches are sized by the tokens of the call
    s = Setup(lens, nq, 8, 2, 128, "bf16", 16, prefix=prefix, seed=42)
    s.most["max_q_len"] = 1 << 24
    s.cache.reserve(s.total, s.most["max_q_len"], max(lens), prefix)
    assert all(x * y * z <= 2048 for x, y, z, _ in H.captured_launches(lambda: s.run()))
    s.run().check()


# ---- append -------------------------------------------------------------------------------------------------------------------

def append_case(dtype, d, hq, hkv, page, lens, nq, rot, pairs, seed, max_pages=None, one=False, positions=True, with_q=True, in_place=False, bad=False):
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    nb, total = len(lens), sum(nq)
    max_pages = max_pages or max(-(-(a + b) // page) for a, b in zip(lens, nq)) + 1
    n_pages = nb * max_pages + 1
    table = torch.randperm(n_pages, generator=g)[:nb * max_pages].view(nb, max_pages).int()
    if bad:
        table[0, 0], table[-1, 0] = -1, n_pages
    kp, vp = (torch.randn((n_pages, hkv, page, d), generator=g).to(dt) for _ in range(2))
    qkv = torch.randn((total + 1, (hq + 2 * hkv) * d + 16), generator=g).to(dt).to(DEV)       # a stride that is no sum of heads
    q, k, v = (x.unflatten(1, (-1, d))[:total] for x in qkv[:, :(hq + 2 * hkv) * d].split([hq * d, hkv * d, hkv * d], 1))
    pos = torch.randint(-3, 60, (total,), generator=g).int() if positions else None
    n_pos = 50
    ang = torch.rand((n_pos, max(rot, 2) // 2), generator=g, dtype=torch.float64) * 7
    rt = torch.cat([ang.cos(), ang.sin()], 1).float() if rot else None
    offs = np.concatenate([[0], np.cumsum(nq)]).tolist()
    p = cd.make_paged_params(dtype=dt, batch=nb, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=n_pages, max_pages=max_pages,
                             rot_dim=rot, rot_pairs=pairs)
    c = cd.PagedCache(p, kp.to(DEV), vp.to(DEV), table.to(DEV), ints(lens))
    if in_place:
        q = q.contiguous()
    q_in = q.clone()
    q_out = q if in_place else torch.empty((total, hq, d), dtype=dt, device=DEV)
    new_lens = None if in_place else ints([0] * nb)
    c.append(k, v, q=q if with_q else None, q_out=q_out if with_q else None, new_offsets=None if one else ints(offs), max_new=max(max(nq), 1),
             positions=None if pos is None else pos.to(DEV), rot_table=None if rt is None else rt.to(DEV), new_lens=new_lens)
    torch.cuda.synchronize()
    f = lambda t: t.float().cpu().numpy()
    wk, wv, wl, wq = ref.append(f(kp), f(vp), table.numpy(), lens, f(q_in), f(k), f(v), offs, None if pos is None else pos.numpy(),
                                None if rt is None else rt.numpy(), rot, pairs, page)
    # two fp32 products and their sum (3 2^-24 (|x| + |y|)), rounded once; values that were not turned are copies
    eps = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    big = float(max(f(qkv).__abs__().max(), 1))
    close = lambda got, want: np.abs(f(got) - want) <= eps * np.abs(want) + (6 * big * 2.0 ** -24) * (np.abs(want) != np.abs(f(got)))
    assert close(c.k_pages, wk).all() and (f(c.v_pages) == wv).all()
    if with_q:
        assert close(q_out, wq).all()
    got_lens = c.cache_lens if in_place else new_lens
    assert got_lens.tolist() == list(wl)
    if not in_place:
        assert c.cache_lens.tolist() == list(lens)
    assert torch.equal(k, qkv[:total, hq * d:(hq + hkv) * d].unflatten(1, (-1, d)))


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 128])
def test_append_rotations(dtype, d, pairs, rot):
    if rot <= d:
        append_case(dtype, d, 6, 2, 16, [0, 5, 15, 16, 31, 40], [1] * 6, rot, pairs, 20, one=True)
        append_case(dtype, d, 6, 2, 16, [0, 5, 15, 16, 31, 40], [3, 0, 1, 30, 7, 4], rot, pairs, 21)


@pytest.mark.parametrize("page", [1, 3, 16, 50])
@pytest.mark.parametrize("hq,hkv", HEADS)
def test_append_pages_and_heads(page, hq, hkv):
    append_case("bf16", 64, hq, hkv, page, [0, 9, 33], [40, 2, 5], 64, "halves", 22)


@pytest.mark.parametrize("nq", [[1, 1, 1], [3, 4, 2], [20, 0, 9]])
def test_append_grows_the_lengths_in_place(nq):
    append_case("bf16", 128, 8, 2, 16, [5, 0, 16], nq, 128, "halves", 23, in_place=True)
    append_case("fp32", 64, 8, 2, 16, [5, 0, 16], nq, 32, "neighbours", 24, in_place=True, positions=False)


def test_append_leaves_full_sequences_and_unnamed_pages():
    # 2 pages of 16: the first sequence is full, the second becomes full, the third lacks one row, the fourth has a length of rubbish
    for nq in ([1, 1, 1, 1], [4, 4, 4, 4], [9, 3, 9, 9]):
        append_case("bf16", 64, 4, 2, 16, [32, 32 - nq[1], 33 - nq[2], -4], nq, 64, "halves", 25, max_pages=2)
    append_case("bf16", 64, 4, 2, 16, [0, 3, 0], [20, 2, 4], 64, "halves", 26, bad=True)


def test_append_without_queries_or_positions():
    append_case("bf16", 128, 8, 2, 16, [5, 0, 16], [3, 1, 2], 64, "neighbours", 27, with_q=False, positions=False)
    append_case("fp32", 64, 8, 2, 16, [5, 0, 16], [1, 1, 1], 0, "halves", 28, one=True, with_q=False, positions=False)


def test_append_of_nothing():
    s = Setup([3, 4], [1, 1], 4, 2, 64, "bf16", 16)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    new_lens = ints([9, 9])
    s.cache.append(none, none, new_offsets=ints([0, 0, 0]), new_lens=new_lens)
    assert new_lens.tolist() == [3, 4]
    s.cache.append(none, none, new_offsets=ints([0, 0, 0]), max_new=50)
    assert s.cache.cache_lens.tolist() == [3, 4]


@pytest.mark.parametrize("bound,offsets,rows", [
    (None, [0, 3, 3, 12], [(0, 3), (3, 0), (3, 9)]),                    # no bound given: every token
    (2, [0, 3, 3, 12], [(0, 2), (3, 0), (3, 2)]),                       # below the tokens of a sequence: its first ones
    (12, [0, 2, 1, 1 << 30], [(0, 2), (2, 0), (1, 11)]),                # falling, and beyond the tokens: what is in range
    (12, [-9, 2, -5, 4], [(0, 2), (2, 0), (0, 4)])])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_bounds_and_offsets(bound, offsets, rows, in_place):
    nb, hq, hkv, d, page, lens = 3, 4, 2, 64, 16, [5, 0, 16]
    g = torch.Generator(device=DEV).manual_seed(39)
    k, v, q = (torch.randn((12, h, d), generator=g, device=DEV) for h in (hkv, hkv, hq))
    p = cd.make_paged_params(dtype="fp32", batch=nb, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=9, max_pages=3)
    c = cd.PagedCache(p, torch.zeros((9, hkv, page, d), device=DEV), torch.zeros((9, hkv, page, d), device=DEV),
                      torch.arange(9, dtype=torch.int32, device=DEV).view(3, 3), ints(lens))
    q_out, new_lens = torch.full_like(q, 77.0), None if in_place else ints([0] * nb)
    c.append(k, v, q=q, q_out=q_out, new_offsets=ints(offsets), max_new=bound, new_lens=new_lens)
    want_k, want_v, want_q = torch.zeros_like(c.k_pages), torch.zeros_like(c.v_pages), torch.full_like(q, 77.0)
    for b, (first, n) in enumerate(rows):
        want_q[first:first + n] = q[first:first + n]
        for t in range(n):
            r = lens[b] + t
            want_k[3 * b + r // page, :, r % page], want_v[3 * b + r // page, :, r % page] = k[first + t], v[first + t]
    assert torch.equal(c.k_pages, want_k) and torch.equal(c.v_pages, want_v) and torch.equal(q_out, want_q)
    assert (c.cache_lens if in_place else new_lens).tolist() == [n + r[1] for n, r in zip(lens, rows)]


# ---- together ---------------------------------------------------------------------------------------------------------------------

def rope(n, d):
    ang = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))
    return torch.cat([ang.cos(), ang.sin()], 1).float().to(DEV)


def test_prompt_then_compression_then_decode():
    """A prompt kept in one page per sequence: rotated and appended, attended, compressed with the attention's normalisers,
    and the compressed cache grown by rotated rows as a paged cache of one page per sequence."""
    n, nb, hq, hkv, d, w, budget = 384, 2, 8, 2, 64, 16, 96
    g = torch.Generator(device=DEV).manual_seed(30)
    dt = torch.float32
    p = cd.make_paged_params(dtype=dt, batch=nb, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=n, n_pages=nb, max_pages=1, rot_dim=d)
    pages = [torch.zeros((nb, hkv, n, d), device=DEV) for _ in range(2)]
    c = cd.PagedCache(p, *pages, ints([[0], [1]]), ints([0, 0]))
    c.reserve(nb * n, n, n)
    q, k, v = (torch.randn((nb * n, h, d), generator=g, device=DEV) for h in (hq, hkv, hkv))
    offs, table = ints([0, n, 2 * n]), rope(n + 8, d)
    q_rot, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((nb * n, hq), device=DEV)
    c.append(k, v, q=q, q_out=q_rot, new_offsets=offs, max_new=n, rot_table=table)
    c.attend(q_rot, out, lse, q_offsets=offs, max_q_len=n, max_cache_len=n)
    cp = cd.make_params(dtype=dt, batch=nb, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, window=w, budget=budget, pool_kernel=5,
                        theta1=-math.inf, theta2=-math.inf)
    win = q_rot.view(nb, n, hq, d)[:, n - w:].transpose(1, 2).contiguous()
    win_lse = lse.view(nb, n, hq)[:, n - w:].transpose(1, 2).contiguous()
    bufs, plain = (cd.CompressBuffers(cp, [n] * nb, DEV, extra_capacity=8) for _ in range(2))
    bufs.compress(win, c.k_pages, c.v_pages, offs, win_lse=win_lse)
    plain.compress(win, c.k_pages, c.v_pages, offs)
    torch.cuda.synchronize()
    assert torch.equal(bufs.indices, plain.indices) and torch.equal(bufs.k_c, plain.k_c)
    # the compressed caches as pages of their capacity; the new token stands at position n of the text
    cap = bufs.cap
    grown = bufs.paged(rot_dim=d)
    grown.reserve(nb, 1, cap)
    for t in range(3):
        q1, k1, v1 = (torch.randn((nb, h, d), generator=g, device=DEV) for h in (hq, hkv, hkv))
        turned = torch.empty_like(q1)
        grown.append(k1, v1, q=q1, q_out=turned, positions=ints([n + t] * nb), rot_table=table)
        o1, l1 = torch.empty_like(q1), torch.empty((nb, hq), device=DEV)
        grown.attend(turned, o1, l1)
        bufs.decode(turned)
        torch.cuda.synchronize()
        assert bufs.cache_lens.tolist() == [budget + t + 1] * nb
        assert (bufs.a_lse - l1).abs().max() < 1e-4
        # Eq. 1 of decode undone: its output is the paged one joined with the calibration state
        a = torch.sigmoid(bufs.c_lse - bufs.a_lse)[..., None]
        assert ((1 - a) * o1 + a * bufs.c_out - bufs.out).abs().max() < 1e-4
        want_k = torch.cat([k1[..., :d // 2] * table[n + t, :d // 2] - k1[..., d // 2:] * table[n + t, d // 2:],
                            k1[..., d // 2:] * table[n + t, :d // 2] + k1[..., :d // 2] * table[n + t, d // 2:]], -1)
        assert (bufs.k_c.view(nb, hkv, cap, d)[:, :, budget + t] - want_k).abs().max() < 1e-5


@pytest.mark.parametrize("prefix", [0, 90])
def test_functions_of_the_module_and_the_cache_agree(prefix):
    s, t = (Setup([70, 33, 9], [3, 1, 2], 8, 2, 64, "bf16", 16, prefix=prefix, seed=43) for _ in range(2))
    new = [torch.randn((3, 2, 64), generator=torch.Generator().manual_seed(44)).bfloat16().to(DEV) for _ in range(2)]
    a, b = s.cache, t.cache
    a.append(*new)
    cd.calidrop_paged_append(b.p, None, 0, new[0], 128, new[1], 128, None, 3, 1, None, None, 0, b.k_pages, b.v_pages, b.page_table, b.cache_lens,
                             b.cache_lens, None)
    a.cache_lens -= 1                                       # the same queries at their own rows again
    b.cache_lens -= 1
    s.run()
    head, tail = (t.qd, t.q_off, t.total, 3, b.k_pages, b.v_pages), (b.page_table, b.cache_lens, 70, t.out, t.lse, b.workspace)
    if prefix:
        cd.calidrop_paged_attend_shared(b.p, *head, t.shared_table, prefix, *tail)
    else:
        cd.calidrop_paged_attend(b.p, *head, *tail)
    s.check()
    t.check()
    assert torch.equal(s.out, t.out) and torch.equal(s.lse, t.lse) and a.cache_lens.tolist() == b.cache_lens.tolist() == [70, 33, 9]
    for x, y in ((a.k_pages, b.k_pages), (a.v_pages, b.v_pages)):
        assert torch.equal(x.nan_to_num(0.25), y.nan_to_num(0.25))


@pytest.mark.parametrize("at_once", [1, 200])
def test_decode_after_rows_appended_as_pages_takes_the_form_of_their_number(at_once):
    # 8 KV heads of 400 rows, then of 1000: one launch, then two, as after as many rows appended one by one
    hkv, budget, n, appended = 8, 400, 450, 600
    cp = cd.make_params(dtype="bf16", batch=1, n_q_heads=32, n_kv_heads=hkv, head_dim=128, window=16, budget=budget, pool_kernel=5)
    g = torch.Generator(device=DEV).manual_seed(41)
    win, k, v, q = (torch.randn(s, generator=g, device=DEV).bfloat16() for s in ((1, 32, 16, 128), (1, hkv, n, 128), (1, hkv, n, 128), (1, 32, 128)))
    new = [torch.randn((appended, hkv, 128), generator=g, device=DEV).bfloat16() for _ in range(2)]
    bufs, plain = (cd.CompressBuffers(cp, [n], DEV, extra_capacity=800) for _ in range(2))
    for b in (bufs, plain):
        b.compress(win, k, v, ints([0, n]))
    form = lambda b: H.captured_launches(lambda: b.decode(q))
    assert len(form(bufs)) == 1
    pages = bufs.paged()
    for t in range(0, appended, at_once):
        k1, v1 = (x[t:t + at_once] for x in new)
        pages.append(k1, v1, new_offsets=ints([0, at_once]), max_new=at_once)
        for r in range(at_once):
            plain.append(k1[r:r + 1], v1[r:r + 1])
    assert form(bufs) == form(plain) and len(form(bufs)) == 2
    for b in (bufs, plain):
        b.decode(q)
    torch.cuda.synchronize()
    assert bufs.cache_lens.tolist() == [budget + appended] and torch.equal(bufs.k_c, plain.k_c) and torch.equal(bufs.v_c, plain.v_c)
    assert torch.equal(bufs.out, plain.out) and torch.equal(bufs.a_lse, plain.a_lse)


def decode_steps(steps, graph):
    """A loop of append + attend + attend_shared on the device, eager or replayed; the rows of every step."""
    nb, hq, hkv, d, page = 3, 8, 2, 128, 16
    g = torch.Generator(device=DEV).manual_seed(31)
    kp, vp = (torch.randn((40, hkv, page, d), generator=g, device=DEV).bfloat16() for _ in range(2))
    p = cd.make_paged_params(dtype="bf16", batch=nb, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=40, max_pages=10, rot_dim=d)
    c = cd.PagedCache(p, kp, vp, torch.arange(30, dtype=torch.int32, device=DEV).view(3, 10), ints([70, 0, 15]))
    c.reserve(nb, 1, 160, 150)
    xs = [[torch.randn((nb, h, d), generator=g, device=DEV).bfloat16() for h in (hq, hkv, hkv)] for _ in range(steps)]
    q, k, v = (x.clone() for x in xs[0])
    turned, out, lse = torch.empty_like(q), torch.empty((2,) + q.shape, dtype=q.dtype, device=DEV), torch.empty((2, nb, hq), device=DEV)
    table, prefix = rope(200, d), torch.arange(30, 40, dtype=torch.int32, device=DEV)

    def step():
        c.append(k, v, q=q, q_out=turned, rot_table=table)
        c.attend(turned, out[0], lse[0])
        c.attend_shared(turned, out[1], lse[1], prefix, 150)
    if graph:
        step()                                              # warm up, then put everything back
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step()
        g2 = torch.Generator(device=DEV).manual_seed(31)
        for t in (kp, vp):
            t.copy_(torch.randn((40, hkv, page, d), generator=g2, device=DEV).bfloat16())
        c.cache_lens.copy_(ints([70, 0, 15]))
    got = []
    for x in xs:
        for dst, src in zip((q, k, v), x):
            dst.copy_(src)
        gr.replay() if graph else step()
        got.append([t.clone() for t in (turned, out, lse, c.cache_lens)])
        torch.cuda.synchronize()
    return got + [[kp, vp]]


def test_a_captured_step_replays_to_the_eager_results():
    for eager, replayed in zip(decode_steps(20, False), decode_steps(20, True)):
        for a, b in zip(eager, replayed):
            assert torch.equal(a, b)


@pytest.mark.parametrize("lens,nq,prefix", [([5000, 300, 2000], [1, 1, 1], 0), ([6000, 900], [40, 30], 0), ([300, 40], [3, 30], 2000)])
def test_a_captured_call_follows_the_lengths(lens, nq, prefix):
    # the lengths are read on the device: replays after they have changed, with eager work between, give what eager calls give
    s = Setup(lens, nq, 8, 2, 128, "bf16", 16, prefix=prefix, seed=37)
    s.cache.k_pages.nan_to_num_(0.5), s.cache.v_pages.nan_to_num_(0.5)         # shorter caches end elsewhere
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for cut in ([0] * 3, [10, 0, 1], [900, 35, 1999], [0, 7, 3], [1, 1, 1]):
        s.cache.cache_lens.copy_(ints([n - c for n, c in zip(lens, cut)]))
        s.run()
        torch.cuda.synchronize()
        eager = s.out.clone(), s.lse.clone()
        s.out.fill_(77), s.lse.fill_(77)
        s.cache.workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.out, eager[0]) and torch.equal(s.lse, eager[1])


def test_results_do_not_depend_on_the_run():
    s = Setup([3000, 200, 900], [2, 1, 4], 8, 2, 128, "bf16", 16, prefix=700, seed=32).run()
    torch.cuda.synchronize()
    first = s.out.clone(), s.lse.clone()
    for _ in range(3):
        s.out.fill_(77), s.lse.fill_(77)
        s.run()
        torch.cuda.synchronize()
        assert torch.equal(s.out, first[0]) and torch.equal(s.lse, first[1])


def test_calls_on_two_streams_with_a_workspace_each():
    a, b = (Setup([3000, 200, 900], [2, 1, 4], 8, 2, 128, "bf16", 16, seed=s) for s in (33, 34))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for s, st in zip((a, b), streams):
            s.run(stream=st)
    a.check()
    b.check()


@pytest.mark.parametrize("by_argument", [True, False])
@pytest.mark.parametrize("prefix", [0, 300])
def test_a_larger_reservation_leaves_a_running_call_its_workspace(prefix, by_argument):
    s = Setup([3000, 200, 900], [2, 1, 4], 8, 2, 128, "bf16", 16, prefix=prefix, seed=40)
    size, old = s.cache.workspace.nbytes, s.cache.workspace.data_ptr()
    x = torch.randn((4096, 4096), device=DEV)
    more = (4 * s.total, 400, 3000) + ((prefix,) if prefix else ())
    need = (cd.calidrop_paged_attend_shared_workspace_bytes if prefix else cd.calidrop_paged_attend_workspace_bytes)(s.cache.p, *more)
    assert need > size
    cached = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (need,) + 4 * (size,)]     # so that nothing below waits for memory
    del cached
    torch.cuda.synchronize()
    side, ended = torch.cuda.Stream(), torch.cuda.Event()
    with torch.cuda.stream(side):
        for _ in range(100):
            x = x @ x / 64                                   # the call behind these starts when everything below is done
        if not by_argument:
            s.run()
    if by_argument:
        s.run(stream=side)
    ended.record(side)
    s.cache.reserve(*more)
    taken = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)]
    early = not ended.query()
    assert all(t.data_ptr() + size <= old or old + size <= t.data_ptr() for t in taken)
    s.check()
    assert early                                             # the call was still ahead when its memory could have been taken


def test_a_workspace_of_the_largest_call_serves_the_others():
    s = Setup([2000, 100], [3, 1], 8, 2, 64, "bf16", 16, seed=35)
    s.cache.workspace = None
    with pytest.raises(cd.CalidropError, match="workspace"):
        s.run()
    s.cache.reserve(500, 400, 2000)
    s.run().check()


def test_pages_past_four_gib():
    # rows whose offsets do not fit 32 bits, in elements and in bytes
    d, hkv, page = 128, 8, 64
    n_pages = 40000                                          # 2.6e9 elements in K
    k, v = (torch.empty((n_pages, hkv, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    s = Setup([150, 90], [100, 1], 16, hkv, d, "bf16", page, seed=36)
    table = [[n_pages - 1 - e if 0 <= e < s.n_pages else e for e in row] for row in s.table]
    for e in range(s.n_pages):
        k[n_pages - 1 - e] = s.cache.k_pages[e]
        v[n_pages - 1 - e] = s.cache.v_pages[e]
    p = cd.make_paged_params(dtype="bf16", batch=2, n_q_heads=16, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=n_pages, max_pages=s.max_pages)
    ws = s.cache.workspace
    s.cache = cd.PagedCache(p, k, v, ints(table), s.cache.cache_lens)
    s.cache.workspace = ws
    s.run().check()
    new = torch.randn((2, hkv, d), device=DEV).bfloat16()
    s.cache.append(new, -new)
    torch.cuda.synchronize()
    assert torch.equal(k[table[0][150 // page], :, 150 % page], new[0]) and torch.equal(v[table[1][90 // page], :, 90 % page], -new[1])
