"""The calls on a cache in pages as far as they need no GPU: the reference against library attention and hand-made values,
the arithmetic of the page lookup, workspace sizes, and what the library and the binding refuse."""
import ctypes
import random

import numpy as np
import pytest
import torch

from oracle import paged_ref as ref
from paper_2507_19906_amd import binding as cd

A = 4096        # an aligned address that no refused call touches


def params(**kw):
    base = dict(dtype="bf16", batch=3, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, n_pages=100, max_pages=20)
    base.update(kw)
    return cd.make_paged_params(**base)


# ---- the reference ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (5, 2), (64, 0), (7, 100)])
def test_reference_attention_is_masked_library_attention(window, sinks):
    g = torch.Generator().manual_seed(1)
    n, rows, Hq, Hkv, D = 6, 23, 4, 2, 16
    q, k, v = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((n, Hq, D), (rows, Hkv, D), (rows, Hkv, D)))
    pos = np.arange(rows - n, rows)
    got = ref.attend(q.numpy(), k.numpy(), v.numpy(), pos, D ** -0.5, window, sinks)
    mask = torch.zeros(n, rows, dtype=torch.bool)
    for t in range(n):
        for j in range(rows):
            i = rows - n + t
            mask[t, j] = j <= i and (window == 0 or j > i - window or j < sinks)
    kk, vv = (x.repeat_interleave(Hq // Hkv, 1).transpose(0, 1) for x in (k, v))
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), kk, vv, attn_mask=mask)
    np.testing.assert_allclose(got["out"], want.transpose(0, 1).numpy(), atol=1e-12)
    z = (q.transpose(0, 1) @ kk.transpose(1, 2) * D ** -0.5).masked_fill(~mask, -np.inf)
    np.testing.assert_allclose(got["lse"], torch.logsumexp(z, -1).t().numpy(), atol=1e-12)
    assert (got["seen"] == mask.sum(1).numpy()).all()


def test_reference_prefix_is_attention_over_both():
    g = np.random.default_rng(2)
    q, k, v = g.normal(size=(3, 4, 8)), g.normal(size=(14, 2, 8)), g.normal(size=(14, 2, 8))
    one = ref.attend(q, k, v, [9 + 2, 9 + 3, 9 + 4], 0.3)                 # one context of 14 rows
    two = ref.attend(q, k, v, [2, 3, 4], 0.3, prefix=9)                   # 9 shared rows ahead of 5 own ones
    for name in ("out", "lse", "seen"):
        np.testing.assert_array_equal(one[name], two[name])
    empty = ref.attend(q, k[:9], v[:9], [-1, -1, -1], 0.3)
    assert (empty["lse"] == -np.inf).all() and (empty["out"] == 0).all()


def test_reference_append_by_hand():
    pages = np.zeros((3, 1, 2, 4))
    table = np.array([[2, 0], [1, -1]])
    k = np.arange(1.0, 13.0).reshape(3, 1, 4)
    turn = np.array([[1.0, 1.0, 0.0, 0.0], [0.0, 0.0, 1.0, 1.0]])         # angle 0, angle 90 degrees
    kp, vp, lens, q = ref.append(pages, pages, table, [1, 2], k, k, -k, [0, 2, 3], [0, 1, 7], turn, 4, "halves", 2)
    assert lens.tolist() == [3, 3]
    assert kp[2, 0, 1].tolist() == [1, 2, 3, 4] and kp[0, 0, 0].tolist() == [-7, -8, 5, 6]
    assert vp[0, 0, 0].tolist() == [-5, -6, -7, -8] and not kp[1].any()  # sequence 1: no page for row 2
    assert q[2, 0].tolist() == [-11, -12, 9, 10]
    assert ref.rotate(k[0], [0.0, 0.0], [1.0, 1.0], 4, "neighbours")[0].tolist() == [-2, 1, -4, 3]
    kept = ref.append(pages, pages, table, [3, 0], k, k, -k, [0, 2, 3], None, turn, 4, "halves", 2)
    assert kept[2].tolist() == [3, 1] and not kept[0][0].any()            # 5 rows do not fit 2 pages of 2


# ---- arithmetic -----------------------------------------------------------------------------------------------

def divide(x, d):
    """The kernels' quotient: one 64-bit product with ceil(2^shift / d), shift = 31 + ceil(log2 d)."""
    shift = 31 + (d - 1).bit_length()
    magic = -(-(1 << shift) // d)
    assert magic < 1 << 32 and x * magic < 1 << 64
    return x * magic >> shift


def test_page_of_a_row_is_exact():
    rng = random.Random(5)
    sizes = [*range(1, 600), 1 << 16, (1 << 16) + 1, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, (1 << 31) - 1, *(rng.randrange(1, 1 << 31) for _ in range(2000))]
    for d in sizes:
        for x in [0, 1, (1 << 31) - 1, 1 << 30, rng.randrange(1 << 31)] + [y for m in (1, 2, rng.randrange(1, (1 << 31) // d + 1))
                                                                          for y in (m * d - 1, m * d, m * d + 1)]:
            if 0 <= x < 1 << 31:
                assert divide(x, d) == x // d


@pytest.mark.parametrize("kw", [{}, dict(batch=64), dict(dtype="fp32", head_dim=64, n_q_heads=8, n_kv_heads=2), dict(n_q_heads=16, n_kv_heads=1),
                                dict(window=100, sinks=4), dict(batch=1, n_kv_heads=32)])
def test_workspace_sizes_do_not_fall(kw):
    p = params(max_pages=1 << 20, **kw)
    rng = random.Random(6)
    for _ in range(3000):
        lo = [rng.randint(0, 1 << rng.randint(0, 14)), rng.randint(1, 1 << rng.randint(0, 14)), rng.randint(0, 1 << rng.randint(0, 17)),
              rng.randint(1, 1 << rng.randint(0, 17))]
        hi = [x + rng.choice([0, 1, rng.randint(0, x)]) for x in lo]
        assert 256 <= cd.calidrop_paged_attend_workspace_bytes(p, *lo[:3]) <= cd.calidrop_paged_attend_workspace_bytes(p, *hi[:3])
        if not p.window:
            assert 256 <= cd.calidrop_paged_attend_shared_workspace_bytes(p, *lo) <= cd.calidrop_paged_attend_shared_workspace_bytes(p, *hi)


# ---- refusals ----------------------------------------------------------------------------------------------------

BAD_PARAMS = [
    (dict(dtype=2), cd.EUNSUPPORTED), (dict(batch=0), cd.EINVAL), (dict(batch=65536), cd.EUNSUPPORTED), (dict(n_q_heads=0), cd.EINVAL),
    (dict(n_q_heads=33), cd.ESHAPE), (dict(n_q_heads=17, n_kv_heads=1), cd.EUNSUPPORTED), (dict(head_dim=96), cd.EUNSUPPORTED),
    (dict(page_size=0), cd.EINVAL), (dict(n_pages=0), cd.EINVAL), (dict(max_pages=0), cd.EINVAL), (dict(n_pages=1 << 25), cd.EUNSUPPORTED),
    (dict(max_pages=1 << 27), cd.EUNSUPPORTED),
    (dict(scale=-1.0), cd.EINVAL), (dict(scale=float("nan")), cd.EINVAL), (dict(scale=float("inf")), cd.EINVAL), (dict(window=-1), cd.EINVAL),
    (dict(sinks=-1), cd.EINVAL), (dict(rot_dim=-16), cd.EINVAL), (dict(rot_dim=144), cd.EINVAL), (dict(rot_dim=24), cd.EUNSUPPORTED),
    (dict(rot_pairs=2), cd.EINVAL)]


def append_args(**kw):
    a = dict(q=A, q_stride=4096, k=A, k_stride=1024, v=A, v_stride=1024, new_offsets=A, total_new=7, max_new=3, positions=A, rot_table=A,
             n_positions=100, k_pages=A, v_pages=A, page_table=A, cache_lens=A, new_lens=A, q_out=2 * A, stream=None)
    a.update(kw)
    return list(a.values())


def attend_args(**kw):
    a = dict(q=A, q_offsets=A, total_q=7, max_q_len=3, k_pages=A, v_pages=A, page_table=A, cache_lens=A, max_cache_len=300, out=A, lse=A,
             workspace=A, workspace_bytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


def shared_args(**kw):
    a = dict(q=A, q_offsets=A, total_q=7, max_q_len=3, k_pages=A, v_pages=A, shared_table=A, shared_len=50, page_table=A, cache_lens=A,
             max_cache_len=300, out=A, lse=A, workspace=A, workspace_bytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


CALLS = [("calidrop_paged_append", append_args), ("calidrop_paged_attend", attend_args), ("calidrop_paged_attend_shared", shared_args)]


@pytest.mark.parametrize("kw,code", BAD_PARAMS)
def test_bad_parameters_are_refused_by_every_call(kw, code):
    p = params(**kw)
    for name, args in CALLS:
        assert getattr(cd.lib(), name)(ctypes.byref(p), *args()) == code, name
        assert cd.calidrop_last_error()
    with pytest.raises(cd.CalidropError):
        cd.calidrop_paged_attend_workspace_bytes(p, 7, 3, 100)
    with pytest.raises(cd.CalidropError):
        cd.calidrop_paged_attend_shared_workspace_bytes(p, 7, 3, 100, 10)


def test_foreign_struct_sizes_are_refused():
    p = params()
    p.struct_size -= 4
    for name, args in CALLS:
        assert getattr(cd.lib(), name)(ctypes.byref(p), *args()) == cd.EINVAL
        assert getattr(cd.lib(), name)(None, *args()) == cd.EINVAL


@pytest.mark.parametrize("name,args,kw,code", [
    *[("calidrop_paged_append", append_args, {n: None}, cd.EINVAL) for n in ("k", "v", "k_pages", "v_pages", "page_table", "cache_lens", "new_lens",
                                                                          "q", "q_out", "rot_table")],
    *[("calidrop_paged_append", append_args, {n: A + 4}, cd.EALIGN) for n in ("q", "k", "v", "k_pages", "v_pages", "page_table", "cache_lens",
                                                                           "new_lens", "q_out", "new_offsets", "positions", "rot_table")],
    ("calidrop_paged_append", append_args, dict(total_new=-1), cd.ESHAPE), ("calidrop_paged_append", append_args, dict(max_new=0), cd.ESHAPE),
    ("calidrop_paged_append", append_args, dict(new_offsets=None), cd.ESHAPE), ("calidrop_paged_append", append_args, dict(n_positions=0), cd.ESHAPE),
    ("calidrop_paged_append", append_args, dict(total_new=(1 << 30) + 1), cd.EUNSUPPORTED), ("calidrop_paged_append", append_args, dict(max_new=(1 << 25) + 1), cd.EUNSUPPORTED),
    *[(c, a, dict(max_q_len=1 << 25), cd.EUNSUPPORTED) for c, a in CALLS[1:]],
    ("calidrop_paged_append", append_args, dict(q_stride=4095), cd.ESHAPE), ("calidrop_paged_append", append_args, dict(k_stride=1023), cd.ESHAPE),
    ("calidrop_paged_append", append_args, dict(v_stride=1025), cd.EALIGN), ("calidrop_paged_append", append_args, dict(q_out=A, q_stride=5120), cd.ESHAPE),
    *[("calidrop_paged_attend", attend_args, {n: None}, cd.EINVAL) for n in ("q", "k_pages", "v_pages", "page_table", "cache_lens", "out", "lse")],
    *[("calidrop_paged_attend", attend_args, {n: A + 8}, cd.EALIGN) for n in ("q", "q_offsets", "k_pages", "v_pages", "page_table", "cache_lens",
                                                                           "out", "lse", "workspace")],
    *[(c, a, dict(workspace=None), cd.EWORKSPACE) for c, a in CALLS[1:]],
    *[(c, a, dict(workspace_bytes=255), cd.EWORKSPACE) for c, a in CALLS[1:]],
    *[(c, a, dict(total_q=-1), cd.ESHAPE) for c, a in CALLS[1:]], *[(c, a, dict(max_q_len=0), cd.ESHAPE) for c, a in CALLS[1:]],
    *[(c, a, dict(max_cache_len=-1), cd.ESHAPE) for c, a in CALLS[1:]], *[(c, a, dict(max_cache_len=321), cd.ESHAPE) for c, a in CALLS[1:]],
    *[(c, a, dict(q_offsets=None), cd.ESHAPE) for c, a in CALLS[1:]],
    *[(c, a, dict(total_q=(1 << 25) + 1), cd.EUNSUPPORTED) for c, a in CALLS[1:]],
    ("calidrop_paged_attend_shared", shared_args, dict(shared_table=None), cd.EINVAL),
    ("calidrop_paged_attend_shared", shared_args, dict(shared_table=A + 4), cd.EALIGN),
    ("calidrop_paged_attend_shared", shared_args, dict(shared_len=0), cd.ESHAPE)])
def test_bad_arguments_are_refused(name, args, kw, code):
    assert getattr(cd.lib(), name)(ctypes.byref(params(rot_dim=64)), *args(**kw)) == code
    assert cd.calidrop_last_error()


def test_a_shared_prefix_goes_without_a_window():
    for kw in (dict(window=5), dict(sinks=3)):
        assert cd.lib().calidrop_paged_attend_shared(ctypes.byref(params(**kw)), *shared_args()) == cd.EUNSUPPORTED


def test_a_call_without_queries_is_nothing():
    p = params()
    assert cd.lib().calidrop_paged_attend(ctypes.byref(p), *attend_args(total_q=0, q=None, out=None, lse=None)) == cd.OK
    assert cd.lib().calidrop_paged_attend_shared(ctypes.byref(p), *shared_args(total_q=0, q=None, out=None, lse=None)) == cd.OK


# ---- the binding ------------------------------------------------------------------------------------------------

def cpu_cache(**kw):
    p = params(n_pages=4, max_pages=2, n_q_heads=4, n_kv_heads=2, head_dim=64, batch=2, rot_dim=32, **kw)
    pages = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    return cd.PagedCache(p, pages, pages.clone(), torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


def test_cache_tensors_have_to_fit_the_parameters():
    c = cpu_cache()
    good = [c.k_pages, c.v_pages, c.page_table, c.cache_lens]
    for at, bad in [(0, good[0][:3]), (0, good[0].float()), (1, good[1].transpose(1, 2).contiguous()), (1, good[1].transpose(2, 3).contiguous().transpose(2, 3)),
                    (2, good[2].long()), (2, good[2][:, :1]), (3, torch.zeros(4, dtype=torch.int32)[::2]), (3, good[3][None])]:
        with pytest.raises(ValueError):
            cd.PagedCache(c.p, *[bad if n == at else t for n, t in enumerate(good)])


def test_call_tensors_have_to_fit_the_cache():
    c = cpu_cache()
    bf = torch.bfloat16
    q, k = torch.zeros((2, 4, 64), dtype=bf), torch.zeros((2, 2, 64), dtype=bf)
    lse, table = torch.zeros((2, 4)), torch.zeros((9, 32))
    for kw in (dict(k=k.float()), dict(v=k[:, :1]), dict(v=torch.zeros((2, 64, 2), dtype=bf).transpose(1, 2)), dict(q=q), dict(q_out=q),
               dict(q=q, q_out=q[:1]), dict(positions=torch.zeros(3, dtype=torch.int32)), dict(positions=torch.zeros(2)),
               dict(new_offsets=torch.zeros(2, dtype=torch.int32)), dict(rot_table=table[:, :31]), dict(rot_table=table.double()),
               dict(new_lens=torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            c.append(**{**dict(k=k, v=k, rot_table=table), **kw})
    for kw in (dict(q=q[:, :2]), dict(q=q.float()), dict(out=q[:1]), dict(lse=lse.double()), dict(lse=lse.t().contiguous().t()),
               dict(q_offsets=torch.zeros(4, dtype=torch.int32)), dict(q_offsets=torch.zeros(3, dtype=torch.int64))):
        with pytest.raises(ValueError):
            c.attend(**{**dict(q=q, out=q.clone(), lse=lse), **kw})
        with pytest.raises(ValueError):
            c.attend_shared(**{**dict(q=q, out=q.clone(), lse=lse, shared_table=torch.zeros(2, dtype=torch.int32), shared_len=20), **kw})
    with pytest.raises(ValueError):
        c.attend_shared(q, q.clone(), lse, torch.zeros(2, dtype=torch.int32), 40)


def test_calls_on_a_cache_off_the_current_gpu_are_refused():
    c = cpu_cache()
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        c.attend(q, q.clone(), torch.zeros((2, 4)))


class Recorder:
    """In the library's place: keeps the arguments of each call by name; sizes are the library's."""

    def __init__(self):
        self.calls, self.library = [], cd.lib()

    def __getattr__(self, name):
        return getattr(self.library, name) if name.endswith("_bytes") else lambda *args: self.calls.append((name, args)) or cd.OK


def recorded_cache(monkeypatch, **kw):
    """A cache whose calls end at the recorder: whatever they are given stays on the host."""
    c, lib = cpu_cache(**kw), Recorder()
    monkeypatch.setattr(cd, "_lib", lib)
    monkeypatch.setattr(c, "_on_device", lambda stream: stream)
    return c, lib


def test_without_a_bound_the_tokens_of_a_sequence_are_at_most_all():
    bf = torch.bfloat16
    for total, offsets, want in [(7, torch.tensor([0, 6, 7], dtype=torch.int32), 7), (0, torch.zeros(3, dtype=torch.int32), 1), (2, None, 1)]:
        with pytest.MonkeyPatch.context() as mp:
            c, lib = recorded_cache(mp)
            q, k, lse = torch.zeros((total, 4, 64), dtype=bf), torch.zeros((total, 2, 64), dtype=bf), torch.zeros((total, 4))
            prefix = torch.zeros(2, dtype=torch.int32)
            c.append(k, k, new_offsets=offsets, rot_table=torch.zeros((9, 32)))
            c.attend(q, q.clone(), lse, q_offsets=offsets)
            c.attend_shared(q, q.clone(), lse, prefix, 20, q_offsets=offsets)
            c.append(k, k, new_offsets=offsets, max_new=5, rot_table=torch.zeros((9, 32)))
            c.attend(q, q.clone(), lse, q_offsets=offsets, max_q_len=5)
        # max_new is argument 9 of append, max_q_len argument 4 of both others
        assert [args[9 if name.endswith("append") else 4] for name, args in lib.calls] == [want, want, want, 5, 5]


def test_a_workspace_is_held_for_every_stream_that_uses_it(monkeypatch):
    # the allocator hands freed memory out again on the stream it came from, unless it knows of the others
    c, _ = recorded_cache(monkeypatch)
    q, lse, prefix = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 4)), torch.zeros(2, dtype=torch.int32)
    known = []
    monkeypatch.setattr(cd, "_stream_object", lambda raw, device: raw)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, raw: known.append((t.data_ptr(), raw)))
    c.reserve(2, 1, 32, 20)
    first = c.workspace.data_ptr()
    for stream in (None, 64, 64, None, 64):
        c.attend(q, q.clone(), lse, stream=stream)
    c.attend_shared(q, q.clone(), lse, prefix, 20, stream=128)
    assert known == [(first, None), (first, 64), (first, 128)]            # once each: asking costs as much as a call's checks
    small = c.workspace
    c.reserve(500, 400, 32)
    assert c.workspace is not small and c.workspace.nbytes > small.nbytes
    c.attend(q, q.clone(), lse, stream=64)
    other = torch.empty(1 << 20, dtype=torch.uint8)
    c.workspace = other
    c.attend(q, q.clone(), lse, stream=64)
    assert known[3][1] == 64 and known[3][0] not in (first, other.data_ptr()) and known[4:] == [(other.data_ptr(), 64)]


def test_workspaces_have_to_be_memory_of_the_cache_s_device():
    c = cpu_cache()
    c.workspace = torch.empty(512, dtype=torch.uint8)
    for bad in (torch.empty(512, dtype=torch.uint8)[::2], torch.empty(512, dtype=torch.uint8, device="meta")):
        with pytest.raises(ValueError, match="workspace"):
            c.workspace = bad
    assert c.workspace.nbytes == 512
    c.workspace = None
    assert c.workspace is None


def test_rows_appended_to_compressed_caches_as_pages_are_counted(monkeypatch):
    # decode is told how many rows live, however they were appended
    cp = cd.make_params(dtype="bf16", batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, window=8, budget=30, pool_kernel=5)
    bufs, plain = (cd.CompressBuffers(cp, [100, 90], "cpu", extra_capacity=20) for _ in range(2))
    lib = Recorder()
    monkeypatch.setattr(cd, "_lib", lib)
    monkeypatch.setattr(cd.PagedCache, "_on_device", lambda self, stream: stream)
    pages = [bufs.paged(), bufs.paged(rot_dim=64)]
    one, some = (torch.zeros((n, 2, 64), dtype=torch.bfloat16) for n in (2, 7))
    q, table, offsets = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((9, 64)), torch.tensor([0, 4, 7], dtype=torch.int32)

    def told(b):
        b.decode(q, stream=64)
        return lib.calls[-1][1][0]._obj.budget

    def grow(n, call):
        call()
        for _ in range(n):
            plain.append(one, one, stream=64)
        assert bufs.live_rows == plain.live_rows and told(bufs) == told(plain)

    assert told(bufs) == 30
    grow(1, lambda: pages[0].append(one, one))
    grow(4, lambda: pages[1].append(some, some, new_offsets=offsets, max_new=4, rot_table=table))
    assert told(bufs) == 35
    grow(0, lambda: pages[0].append(one, one, new_lens=torch.zeros(2, dtype=torch.int32)))          # the lengths stay
    grow(1, lambda: pages[0].append(one, one, new_lens=bufs.cache_lens))
    grow(7, lambda: pages[0].append(some, some, new_offsets=offsets))
    grow(7, lambda: pages[0].append(some, some, new_offsets=offsets))
    assert told(bufs) == 50                                           # full
    lib.calidrop_paged_append = lambda *args: cd.EINVAL
    lib.calidrop_last_error = lambda: b"refused"
    bufs._compressed(), plain._compressed()
    with pytest.raises(cd.CalidropError):
        pages[0].append(one, one)
    grow(0, lambda: None)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1), (16, 1), (32, 8)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_calls_behind_a_prefix_launch_fewer_than_2_to_32_threads(dtype, hq, hkv):
    # the joining launch has four rows to a workgroup of 256 threads: 2^26 - 4 rows of a KV head at most
    p = params(dtype=dtype, batch=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=64)
    G = hq // hkv
    for tokens in (1 << 26, (1 << 26) - 1, (1 << 26) - 3, (1 << 26) - 4, (1 << 26) - 16):
        tokens //= G
        for total in {tokens, min(tokens, (1 << 29) // hq)}:
            joined = min(tokens, total) * G                            # no sequence has more tokens than the call
            rows = 128 if dtype == "bf16" else 64                       # of a block
            blocks = (-(-joined // rows) - (-total * G // rows)) * hkv
            args = shared_args(total_q=total, max_q_len=tokens, workspace_bytes=256)
            size = lambda: cd.calidrop_paged_attend_shared_workspace_bytes(p, total, tokens, 300, 50)
            if total * hq > 1 << 29 or (tokens * G + 63) // 64 * hkv > 1 << 23 or -(-joined // 4) >= 1 << 24 or blocks >= 1 << 24:
                assert cd.lib().calidrop_paged_attend_shared(ctypes.byref(p), *args) == cd.EUNSUPPORTED, (tokens, total)
                with pytest.raises(cd.CalidropError, match="2\\^"):
                    size()
            else:
                assert cd.lib().calidrop_paged_attend_shared(ctypes.byref(p), *args) == cd.EWORKSPACE, (tokens, total)
                assert size() > 256


def test_blocks_of_a_prefix_and_of_the_sequences_launch_fewer_than_2_to_32_threads():
    # 2^23 workgroups of each: fp32 blocks of 64 rows behind a prefix as many again; bf16 blocks of 128 are half as many
    for dtype, code in (("fp32", cd.EUNSUPPORTED), ("bf16", cd.EWORKSPACE)):
        p = params(dtype=dtype, batch=1 << 11, n_q_heads=32, n_kv_heads=32, head_dim=64, n_pages=1, max_pages=20)
        args = dict(total_q=1 << 24, max_q_len=1 << 13, workspace_bytes=256)
        assert cd.lib().calidrop_paged_attend_shared(ctypes.byref(p), *shared_args(**args)) == code
        assert cd.lib().calidrop_paged_attend(ctypes.byref(p), *attend_args(**args)) == cd.EWORKSPACE


def test_a_loose_bound_of_the_tokens_needs_a_workspace_but_no_larger_launch():
    p = params(batch=3)
    assert cd.lib().calidrop_paged_attend_shared(ctypes.byref(p), *shared_args(total_q=7, max_q_len=1 << 21, workspace_bytes=256)) == cd.EWORKSPACE


def test_functions_and_cache_hand_the_library_the_same(monkeypatch):
    c, lib = recorded_cache(monkeypatch)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    q, k, v = (torch.zeros((7, h, 64), dtype=torch.bfloat16) for h in (4, 2, 2))
    part = torch.zeros((7, 5, 64), dtype=torch.bfloat16)[:, 1:3]           # of a projection: tokens 320 elements apart
    lse, table, offs, pos, prefix, lens, out = torch.zeros((7, 4)), torch.zeros((9, 32)), i32(3), i32(7), i32(2), i32(2), q.clone()
    c.workspace = torch.empty(1 << 22, dtype=torch.uint8)
    monkeypatch.setattr(c, "_hold", lambda ws, st: None)
    c.append(part, v, q=q, q_out=out, new_offsets=offs, max_new=5, positions=pos, rot_table=table, new_lens=lens, stream=64)
    cd.calidrop_paged_append(c.p, q, 256, part, 320, v, 128, offs, 7, 5, pos, table, 9, c.k_pages, c.v_pages, c.page_table, c.cache_lens, lens, out, 64)
    c.append(k, v, new_offsets=offs, max_new=5, stream=64)
    cd.calidrop_paged_append(c.p, None, 0, k, 128, v, 128, offs, 7, 5, None, None, 0, c.k_pages, c.v_pages, c.page_table, c.cache_lens, c.cache_lens, None, 64)
    c.attend(q, out, lse, q_offsets=offs, max_q_len=6, max_cache_len=30, stream=64)
    cd.calidrop_paged_attend(c.p, q, offs, 7, 6, c.k_pages, c.v_pages, c.page_table, c.cache_lens, 30, out, lse, c.workspace, 64)
    c.attend_shared(q, out, lse, prefix, 20, q_offsets=offs, max_q_len=6, stream=64)
    cd.calidrop_paged_attend_shared(c.p, q, offs, 7, 6, c.k_pages, c.v_pages, prefix, 20, c.page_table, c.cache_lens, 32, out, lse, c.workspace, 64)
    value = lambda x: getattr(x, "value", x)                            # a pointer, however it was wrapped
    for (name, a), (name2, b) in zip(lib.calls[::2], lib.calls[1::2]):
        assert name == name2 and ctypes.addressof(a[0]._obj) == ctypes.addressof(b[0]._obj)
        assert [value(x) for x in a[1:]] == [value(x) for x in b[1:]]
    assert len(lib.calls) == 8
