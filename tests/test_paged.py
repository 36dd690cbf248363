"""The paged cache: append with rotation, attention over bf16 / fp32 / 4-bit pages, read-back, against
plain 64-bit forms (tests/paged_reference.py)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2605_29873_b200 as mkv
from tests import paged_reference as R

BF16, F32, INT4 = mkv.MKV_BF16, mkv.MKV_F32, mkv.MKV_INT4
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
TORCH = {BF16: torch.bfloat16, F32: torch.float32}


# ---------------------------------------------------------------- no GPU needed

def test_page_and_workspace_sizes():
    assert mkv.paged_page_bytes(8, 128, 64, BF16) == 2 * 8 * 64 * 128 * 2
    assert mkv.paged_page_bytes(8, 128, 64, F32) == 2 * 8 * 64 * 128 * 4
    # 4 bits: 64 + 64 bytes of codes and 4 * (2 + 2) * 2 of scales and lowest values per token and head
    assert mkv.paged_page_bytes(8, 128, 64, INT4) == 8 * 64 * (64 + 64 + 32)
    assert mkv.paged_page_bytes(3, 64, 16, INT4) == 3 * 16 * (32 + 32 + 16)
    for bad in [(0, 128, 16, BF16), (1, 96, 16, BF16), (1, 128, 8, BF16), (1, 128, 48, BF16), (1, 128, 512, BF16), (1, 128, 16, 3)]:
        assert mkv.paged_page_bytes(*bad) == 0
    n = mkv.paged_workspace_bytes(32, 8, 128, 16)
    assert n > 0 and n % 256 == 0
    for bad in [(33, 1, 128, 1), (5, 2, 128, 1), (4, 4, 96, 1), (4, 4, 64, 0), (4, 4, 64, 1 << 16)]:
        assert mkv.paged_workspace_bytes(*bad) == 0


def test_create_refuses_bad_arguments():
    lib = mkv.load_library()
    fake, ctx = 1 << 20, C.c_void_p(0)
    ws = mkv.paged_workspace_bytes(8, 2, 128, 4)
    page = mkv.paged_page_bytes(2, 128, 16, BF16)

    def create(**kw):
        a = dict(layers=2, q=8, kv=2, d=128, page=16, n=10, batch=4, kvt=BF16, io=BF16, out=BF16, pages=fake, pb=20 * page,
                 ws=fake, wb=ws, dev=0)
        a.update(kw)
        return lib.mkv_paged_create(a["layers"], a["q"], a["kv"], a["d"], a["page"], a["n"], a["batch"], a["kvt"], a["io"],
                                    a["out"], a["pages"], a["pb"], a["ws"], a["wb"], a["dev"], C.byref(ctx))

    for kw in [dict(layers=0), dict(q=7), dict(n=0), dict(batch=0), dict(kvt=3), dict(io=2), dict(out=2), dict(dev=-1),
               dict(pages=None), dict(pages=fake + 8), dict(pb=20 * page - 1), dict(ws=None),
               dict(io=F32), dict(kvt=INT4, io=F32, out=BF16), dict(kvt=F32), dict(kv=0)]:
        assert create(**kw) == 1, kw
    for kw in [dict(d=96), dict(page=24), dict(page=512), dict(q=66)]:
        assert create(**kw) == 5, kw
    for kw in [dict(ws=fake + 16), dict(wb=ws - 1)]:
        assert create(**kw) == 4, kw
    if not torch.cuda.is_available():
        assert create() == 6
    assert lib.mkv_paged_create(1, 1, 1, 64, 16, 1, 1, 0, 0, 0, fake, page, fake, ws, 0, None) == 1


def test_calls_refuse_a_missing_handle():
    lib = mkv.load_library()
    one = 256
    assert lib.mkv_paged_append(None, 0, one, 128, one, 128, one, 128, one, 1, 1, None, one, one, 1, None, None) == 1
    assert lib.mkv_paged_attend(None, 0, one, 128, one, None, 1, 1, None, 1, one, one, 1, 0.0, 0, None) == 1
    assert lib.mkv_paged_read(None, 0, 1, None, one, one, 1, one, one, 1, None) == 1
    assert lib.mkv_paged_set_rotation(None, None, 0, 0) == 1
    assert lib.mkv_paged_status_sync(None, None) == 1 and lib.mkv_paged_reset(None) == 1
    assert lib.mkv_paged_launch_count(None) == 0
    lib.mkv_paged_destroy(None)


def test_the_handle_needs_a_gpu_tensor():
    with pytest.raises(RuntimeError):
        mkv.PagedKV(torch.zeros(1, 4, 2, 1, 16, 64, dtype=torch.bfloat16), 1, 1, 64, 16, 1)


# ---------------------------------------------------------------- helpers

class Case:
    """A cache whose untouched bytes are all ones (NaN in every format), a batch, and its inputs."""

    def __init__(self, kind, hq, hk, d, page, lens, new=None, layers=1, layer=0, io=None, out=None, seed=0, extra_pages=2,
                 max_batch=None, pad_tokens=0):
        self.kind, self.hq, self.hk, self.d, self.page, self.layer = kind, hq, hk, d, page, layer
        self.io = (F32 if kind == F32 else BF16) if io is None else io
        self.out = self.io if out is None else out
        self.lens_h = list(lens)
        self.new_h = [1 if L else 0 for L in lens] if new is None else list(new)
        self.single = new is None
        B = len(lens)
        g = torch.Generator().manual_seed(seed)
        need = [-(-L // page) for L in lens]
        self.per = max(1, max(need))
        n_pages = sum(need) + extra_pages
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table_h = torch.full((B, self.per), -1, dtype=torch.int32)
        for b in range(B):
            for i in range(need[b]):
                self.table_h[b, i] = order.pop()
        shape = (layers, n_pages, hk, page // 16 * (16 * d + 128 * (d // 32))) if kind == INT4 else (layers, n_pages, 2, hk, page, d)
        nbytes = math.prod(shape) * {INT4: 1, BF16: 2, F32: 4}[kind]
        self.pages = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
        if kind != INT4:
            self.pages = self.pages.view(TORCH[kind])
        self.pages = self.pages.reshape(shape)
        self.ctx = mkv.PagedKV(self.pages, hq, hk, d, page, max_batch or B, kv_dtype=kind, io_dtype=self.io, out_dtype=self.out)
        self.lens = torch.tensor(self.lens_h, dtype=torch.int32, device="cuda")
        self.table = self.table_h.cuda()
        st = [0]
        for n in ([1] * B if self.single else self.new_h):
            st.append(st[-1] + n)
        self.starts_h, self.T = st, st[-1] + pad_tokens
        self.starts = None if self.single else torch.tensor(st, dtype=torch.int32, device="cuda")
        self.gen = torch.Generator(device="cuda").manual_seed(seed + 1)

    def rand(self, *shape, dtype=None):
        return torch.randn(*shape, generator=self.gen, device="cuda").to(dtype or TORCH[self.io])

    def fill(self, kscale=None, vscale=1.0):
        """Appends every sequence's rows [0, lens) without rotation."""
        total = sum(self.lens_h)
        if not total:
            return
        k = (self.rand(total, self.hk, self.d, dtype=torch.float32) * (kscale or 1 / math.sqrt(self.d))).to(TORCH[self.io])
        v = (self.rand(total, self.hk, self.d, dtype=torch.float32) * vscale).to(TORCH[self.io])
        st = torch.tensor([0] + list(np.cumsum(self.lens_h)), dtype=torch.int32, device="cuda")
        self.ctx.append(self.layer, None, k, v, self.lens, self.table, starts=st)

    def tokens(self):
        """(sequence, token row, position) of every new token that has a place."""
        for b, (a, e) in enumerate(zip(self.starts_h, self.starts_h[1:])):
            for i in range(a, e):
                p = self.lens_h[b] - (e - a) + i - a
                if p >= 0:
                    yield b, i, p

    def check_attend(self, e_p, e_k=0.0, e_v=0.0, window=0, scale=0.0, q=None, lse=True, max_new=None, stream=None, table=None):
        q = self.rand(self.T, self.hq, self.d) * 2 if q is None else q
        out = torch.full((self.T, self.hq, self.d), 7.0, dtype=TORCH[self.out], device="cuda")
        ls = torch.full((self.T, self.hq), 7.0, device="cuda") if lse else None
        self.ctx.attend(self.layer, q, self.lens, self.table if table is None else table, out, starts=self.starts,
                        max_new=max_new or max([1] + self.new_h), scale=scale, window=window, lse=ls, stream=stream)
        self.ctx.status_sync()
        torch.cuda.synchronize()
        self.compare(q, out, ls, e_p, e_k, e_v, window, scale)
        return out, ls

    def compare(self, q, out, ls, e_p, e_k=0.0, e_v=0.0, window=0, scale=0.0):
        K, V = R.cache_values(self.pages, self.kind, self.layer, self.d, self.page)
        KS, VS = R.cache_sizes(self.pages, self.kind, self.layer, self.d, self.page)
        for b, (a, e) in enumerate(zip(self.starts_h, self.starts_h[1:])):
            if e == a:
                continue
            L = self.lens_h[b]
            k, v, ks, vs = (R.rows_of(x, self.table_h[b].cuda(), L, self.page) for x in (K, V, KS, VS))
            ref, lse, mean_abs, s_abs = R.attend(q[a:e].double(), k, v, L - (e - a), window, scale, (ks, vs))
            bound = R.out_bound(ref, mean_abs, s_abs, self.d, L, HALF[self.out], e_p, e_k, e_v)
            err = (out[a:e].double() - ref).abs()
            assert torch.isfinite(out[a:e]).all(), f"sequence {b}"
            assert (err <= bound).all(), f"sequence {b}: out off by up to {float((err / bound).max()):.3g} of its bound"
            if ls is not None:
                dead = lse == -math.inf
                assert (ls[a:e][dead] == -math.inf).all()
                err = (ls[a:e].double() - lse).abs()[~dead]
                assert (err <= R.lse_bound(lse, s_abs, self.d, L, e_p, e_k)[~dead]).all(), f"sequence {b}: lse"
        assert (out[self.starts_h[-1]:] == 7).all()
        if ls is not None:
            assert (ls[self.starts_h[-1]:] == 7).all()


# Roundings below 32 bits, by path.  e_p: the weights enter the second product as a sum of two bf16
# (2^-17 of the value is left) over bf16 pages, as one fp16 (2^-11), or a sum of two where out is fp32,
# over 4-bit pages, whose lowest values meet them as a sum of two bf16; as they are over fp32 pages.
# From 65 rows (tokens x group) of a sequence and head on, a tile kernel may take over (bf16 batches: from 25): weights one bf16
# (2^-8) over bf16 pages; over 4-bit pages one fp16, and the rows themselves rounded to fp16 (2^-11), fp32
# queries too (another 2^-11 of every product).
def roundings(kind, out, rows, io=BF16):
    tiles = rows > (24 if kind == BF16 else 64)
    if kind == F32:
        return dict(e_p=0.0)
    if kind == BF16:
        return dict(e_p=2.0 ** -8 if tiles else 2.0 ** -16)
    if tiles:
        return dict(e_p=2.0 ** -11, e_k=2.0 ** (-10 if io == F32 else -11), e_v=2.0 ** -11)
    return dict(e_p=2.0 ** -11 if out == BF16 else 2.0 ** -15)


# ---------------------------------------------------------------- append

APPEND = [
    # kind, io, d, hq, hk, page, lens, new, rot, interleaved, positions
    (BF16, None, 128, 8, 2, 16, [1, 17, 40], None, 128, False, None),
    (BF16, None, 64, 5, 5, 32, [33, 200, 7, 64], [33, 1, 0, 64], 64, True, None),
    (BF16, None, 128, 14, 2, 64, [130, 65], [3, 65], 32, False, "far"),
    (F32, None, 64, 4, 1, 16, [16, 31, 300], [16, 15, 299], 32, True, None),
    (F32, None, 128, 6, 3, 128, [129], [129], 16, False, "far"),
    (INT4, None, 128, 8, 2, 16, [1, 18, 47, 0], None, 128, False, None),
    (INT4, None, 64, 6, 3, 32, [33, 200, 7, 64], [33, 2, 0, 64], 64, True, "far"),
    (INT4, F32, 128, 4, 4, 256, [500, 3], [500, 3], 48, False, None),
    (INT4, BF16, 128, 8, 1, 64, [2000], [1999], 0, False, None),   # more than 1024 tokens, odd offset
    (BF16, None, 128, 2, 1, 64, [1500], [1333], 128, False, None),
    (INT4, BF16, 64, 2, 2, 32, [9001, 8000], [9000, 7997], 64, True, None),   # more than 16384 tokens
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(case):
    kind, io, d, hq, hk, page, lens, new, rot, inter, far = APPEND[case]
    c = Case(kind, hq, hk, d, page, lens, new, layers=2, layer=1, io=io, seed=case, pad_tokens=0 if new is None else 3)
    inv = (10000.0 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32) if rot else np.zeros(0, np.float32)
    c.ctx.set_rotation(inv, interleaved=inter)
    before = c.pages.clone().view(torch.uint8)
    # q, k, v as slices of one buffer
    qkv = c.rand(c.T, hq + 2 * hk, d)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    q_out = torch.full((c.T, hq, d), 7.0, dtype=TORCH[c.io], device="cuda")
    at = torch.zeros(c.T, dtype=torch.long)
    for b, i, p in c.tokens():
        at[i] = p
    positions = None
    if far:
        at = torch.randint(0, 1 << 20, (c.T,), generator=torch.Generator().manual_seed(9))
        positions = at.to(torch.int32).cuda()
    c.ctx.append(1, q, k, v, c.lens, c.table, q_out=q_out, starts=c.starts, positions=positions)
    c.ctx.status_sync()
    at = at.cuda()
    live = [(b, i, p) for b, i, p in c.tokens()]
    rows = torch.tensor([i for _, i, _ in live], device="cuda")
    page_of = torch.tensor([int(c.table_h[b, p // page]) for b, _, p in live], device="cuda")
    row_of = torch.tensor([p % page for _, _, p in live], device="cuda")

    def near(got, want, x):
        # one rounding to the type, and a rotation in 32 bits: cos and sin to 2^-22, three roundings,
        # of products no larger than the head's largest channel
        pair = x.abs().amax(-1, keepdim=True) if rot else x * 0
        assert ((got.double() - want).abs() <= HALF[c.io] * want.abs() + 2.0 ** -20 * pair).all()

    turned = R.rotate(q.double(), at, inv, inter)
    near(q_out[rows], turned[rows], q.double()[rows])
    untouched = torch.ones(c.T, dtype=torch.bool, device="cuda")
    untouched[rows] = False
    assert (q_out[untouched] == 7).all()

    kt = R.rotate(k.double(), at, inv, inter)[rows]
    if kind != INT4:
        got = c.pages[1]
        near(got[page_of, 0, :, row_of], kt, k.double()[rows])
        assert (got[page_of, 1, :, row_of] == v[rows]).all()
    else:
        (kc, ks, kl), (vc, vs, vl) = R.int4_parts(c.pages[1], d, page)
        for (codes, scale, low), x in (((kc, ks, kl), kt), ((vc, vs, vl), v[rows].double())):
            wc, wscale, wlow, t = R.quantise(x)
            assert torch.equal(scale[page_of, :, row_of], wscale) and torch.equal(low[page_of, :, row_of], wlow)
            got = codes[page_of, :, row_of].unflatten(-1, (-1, 32))
            # a rotated key computed in 64 bits may fall on the other side of a border it touches
            border = ((t - t.floor()) - 0.5).abs() < 1e-9 if x is kt else torch.zeros_like(t, dtype=torch.bool)
            assert ((got == wc) | border).all()
    # everything else is as it was
    after = c.pages.clone().view(torch.uint8)
    assert torch.equal(before.reshape(c.pages.shape[0], -1)[0], after.reshape(c.pages.shape[0], -1)[0])
    mark = torch.zeros(c.pages.shape[1], page, dtype=torch.bool, device="cuda")
    mark[page_of, row_of] = True
    if kind != INT4:
        rest = c.pages[1].movedim(-2, 1)[~mark].contiguous().view(torch.uint8)
        assert (rest == 255).all()
    else:
        (kc, ks, kl), (vc, vs, vl) = R.int4_parts(c.pages[1], d, page)
        for codes, scale, low in ((kc, ks, kl), (vc, vs, vl)):
            assert (codes.movedim(-2, 1)[~mark] == 15).all()
            assert torch.isnan(scale.movedim(-2, 1)[~mark]).all() and torch.isnan(low.movedim(-2, 1)[~mark]).all()


@pytest.mark.gpu
def test_append_in_place_and_without_queries():
    c = Case(BF16, 4, 2, 128, 16, [9, 5], [9, 5])
    inv = np.linspace(1, 1e-4, 64).astype(np.float32)
    c.ctx.set_rotation(inv)
    q, k, v = c.rand(14, 4, 128), c.rand(14, 2, 128), c.rand(14, 2, 128)
    apart = torch.zeros_like(q)
    c.ctx.append(0, q, k, v, c.lens, c.table, q_out=apart, starts=c.starts)
    one = c.pages.clone()
    same = q.clone()
    c.ctx.append(0, same, k, v, c.lens, c.table, q_out=same, starts=c.starts)
    c.ctx.append(0, None, k, v, c.lens, c.table, starts=c.starts)
    assert torch.equal(same, apart) and torch.equal(one.view(torch.uint8), c.pages.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("io", [BF16, F32])
def test_int4_special_groups(io):
    """Constant groups are exact, a zero group is zero, a group with a NaN or an infinity becomes NaN and
    leaves its neighbours alone, huge and tiny values keep their scale."""
    c = Case(INT4, 1, 1, 128, 16, [6], [6], io=io)
    x = c.rand(6, 1, 128)
    x[0] = 0
    x[1] = 3.25
    x[2, :, 5] = math.nan
    x[2, :, 70] = math.inf
    x[3, :, 33] = -math.inf
    x[4] *= 1e37
    x[5] *= 1e-36
    c.ctx.append(0, None, x, x, c.lens, c.table, starts=c.starts)
    K, V = torch.zeros(1, 1, 6, 128, dtype=TORCH[io], device="cuda"), torch.zeros(1, 1, 6, 128, dtype=TORCH[io], device="cuda")
    c.ctx.read(0, c.lens, c.table, K, V)
    c.ctx.status_sync()
    assert torch.equal(torch.nan_to_num(K.float(), 99.0), torch.nan_to_num(V.float(), 99.0))
    got = K[0, 0].double()
    assert (got[0] == 0).all() and (got[1] == 3.25).all()
    bad = torch.zeros(6, 4, dtype=torch.bool, device="cuda")
    bad[2, 0] = bad[2, 2] = bad[3, 1] = True
    assert torch.equal(torch.isnan(got).reshape(6, 4, 32), bad[..., None].expand(6, 4, 32))
    g = x[:, 0].double().reshape(6, 4, 32)
    step = (g.amax(-1) - g.amin(-1)) / 15
    # half a step, what the scale's rounding moves the last code by, the lowest value's rounding, the store's
    tol = step * (0.5 + 15 * 2.0 ** -8) + g.amin(-1).abs() * 2.0 ** -8
    err = (got.reshape(6, 4, 32) - g).abs()
    assert (err <= tol[..., None] + HALF[io] * g.abs())[~bad].all()


# ---------------------------------------------------------------- read

@pytest.mark.gpu
@pytest.mark.parametrize("kind,io,d,page", [(BF16, None, 128, 16), (BF16, None, 64, 64), (F32, None, 64, 32), (F32, None, 128, 16),
                                            (INT4, BF16, 128, 64), (INT4, F32, 64, 16), (INT4, BF16, 64, 256)])
def test_read(kind, io, d, page):
    lens = [0, 1, 37, 300]
    c = Case(kind, 2, 2, d, page, lens, io=io, layers=2, layer=1)
    c.fill()
    K, V = R.cache_values(c.pages, kind, 1, d, page)
    for first in (None, [0, 1, 20, 37]):
        k = torch.full((4, 2, 300, d), 7.0, dtype=TORCH[c.io], device="cuda")
        v = torch.full_like(k, 7.0)
        f = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
        c.ctx.read(1, c.lens, c.table, k, v, first=f)
        c.ctx.status_sync()
        for b, L in enumerate(lens):
            a = 0 if first is None else first[b]
            for got, val in ((k, K), (v, V)):
                want = R.rows_of(val, c.table[b], L, page)[:, a:]
                if kind == INT4:   # scale * code + lowest in 32 bits, rounded to the type
                    assert ((got[b, :, : L - a].double() - want).abs() <= (HALF[c.io] + 2.0 ** -22) * want.abs() + 2.0 ** -22).all()
                else:
                    assert torch.equal(got[b, :, : L - a].double(), want)
                assert (got[b, :, L - a:] == 7).all()
    # too few rows: the first ones, and a status
    k = torch.zeros(4, 2, 100, d, dtype=TORCH[c.io], device="cuda")
    v = torch.zeros_like(k)
    c.ctx.read(1, c.lens, c.table, k, v)
    with pytest.raises(mkv.MkvError) as e:
        c.ctx.status_sync()
    assert e.value.code == 3
    c.ctx.reset()
    c.ctx.status_sync()


# ---------------------------------------------------------------- attend

SINGLE = [
    # kind, io, out, d, hq, hk, page, lens, window
    (BF16, None, None, 128, 8, 2, 16, [1, 2, 15, 16, 17, 0, 31, 33, 64, 65, 127, 500], 0),
    (BF16, None, F32, 128, 7, 1, 64, [1000, 3, 0, 777], 0),
    (BF16, None, F32, 128, 16, 2, 32, [1, 700, 1025], 100),
    (BF16, None, None, 64, 6, 3, 128, [129, 1, 4000], 0),
    (BF16, None, F32, 64, 32, 1, 256, [300, 17], 16),
    (BF16, None, F32, 128, 5, 5, 16, [33, 48, 1], 1),
    (BF16, None, F32, 128, 24, 2, 16, [333, 90], 0),
    (BF16, None, None, 128, 32, 1, 16, [5000], 0),
    (F32, None, None, 64, 4, 1, 16, [1, 2, 0, 15, 16, 17, 500], 0),
    (F32, None, None, 128, 24, 3, 64, [1000, 3, 65], 50),
    (F32, None, None, 128, 9, 1, 32, [100], 0),
    (F32, None, None, 64, 64, 2, 32, [100, 2500], 0),
    (INT4, BF16, BF16, 128, 8, 2, 16, [1, 2, 15, 16, 17, 0, 31, 33, 64, 65, 127, 500], 0),
    (INT4, BF16, F32, 128, 7, 1, 64, [1000, 3, 0, 777], 0),
    (INT4, F32, F32, 128, 4, 4, 32, [1, 700, 1025], 100),
    (INT4, BF16, F32, 64, 6, 3, 128, [129, 1, 4000], 0),
    (INT4, F32, F32, 64, 32, 1, 256, [300, 17], 16),
    (INT4, BF16, BF16, 128, 24, 2, 16, [333, 90], 1),
    (INT4, BF16, BF16, 128, 32, 1, 16, [5000], 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(SINGLE)))
def test_attend_single_tokens(case):
    kind, io, out, d, hq, hk, page, lens, window = SINGLE[case]
    c = Case(kind, hq, hk, d, page, lens, io=io, out=out, layers=2, layer=1, seed=case)
    c.fill()
    c.check_attend(window=window, **roundings(kind, c.out, hq // hk))


MANY = [
    # kind, io, out, d, hq, hk, page, lens, new, window
    (BF16, None, None, 128, 8, 2, 16, [5, 64, 100, 0, 3], [5, 1, 7, 0, 0], 0),          # up to 28 rows
    (BF16, None, F32, 128, 4, 2, 64, [500, 40, 17], [9, 3, 17], 30),
    (BF16, None, F32, 64, 7, 7, 32, [130, 9, 300], [8, 9, 2], 0),
    (BF16, None, F32, 128, 8, 1, 16, [90, 200], [8, 5], 4),                                # 64 rows
    (BF16, None, None, 128, 8, 2, 64, [300, 129, 700], [300, 64, 5], 0),                   # tiles
    (BF16, None, F32, 128, 14, 2, 16, [257, 1, 95], [100, 1, 95], 0),
    (BF16, None, F32, 64, 4, 4, 128, [777, 130], [257, 130], 200),
    (BF16, None, F32, 128, 1, 1, 256, [1000], [999], 0),
    (BF16, None, F32, 128, 32, 1, 32, [40, 3], [33, 3], 0),
    (F32, None, None, 64, 4, 1, 16, [50, 200, 33], [50, 7, 0], 0),
    (F32, None, None, 128, 6, 2, 64, [150, 1], [70, 1], 20),
    (INT4, BF16, BF16, 128, 8, 2, 16, [5, 64, 100, 0, 3], [5, 1, 7, 0, 0], 0),
    (INT4, F32, F32, 128, 4, 2, 64, [500, 40, 17], [9, 3, 17], 30),
    (INT4, BF16, F32, 64, 7, 7, 32, [130, 9, 300], [8, 9, 2], 0),
    (INT4, BF16, BF16, 128, 8, 2, 64, [300, 129, 700], [300, 64, 5], 0),
    (INT4, F32, F32, 64, 4, 4, 128, [777, 130], [257, 130], 200),
    (INT4, BF16, F32, 128, 14, 2, 16, [257, 1, 95], [100, 1, 95], 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(MANY)))
def test_attend_several_tokens(case):
    kind, io, out, d, hq, hk, page, lens, new, window = MANY[case]
    c = Case(kind, hq, hk, d, page, lens, new, io=io, out=out, seed=100 + case, pad_tokens=2)
    c.fill()
    c.check_attend(window=window, **roundings(kind, c.out, hq // hk * max(new), c.io))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, F32, INT4])
def test_more_new_tokens_than_the_cache_holds(kind):
    """lens below the number of new tokens: the first ones have no place, see nothing and change nothing."""
    c = Case(kind, 4, 2, 128, 16, [3, 0, 20], [5, 2, 20])
    k, v, q = c.rand(27, 2, 128), c.rand(27, 2, 128), c.rand(27, 4, 128)
    q_out = torch.full_like(q, 7.0)
    c.ctx.append(0, q, k, v, c.lens, c.table, q_out=q_out, starts=c.starts)
    assert (q_out[:2] == 7).all() and (q_out[5:7] == 7).all() and torch.equal(q_out[2:5], q[2:5])
    out, lse = c.check_attend(q=q, **roundings(kind, c.out, 2 * 20))
    assert (out[:2] == 0).all() and (out[5:7] == 0).all() and (lse[:2] == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, F32, INT4])
@pytest.mark.parametrize("new", [3, 90])
def test_what_is_not_seen_has_no_influence(kind, new):
    """Rows that a token does not see hold NaN or infinities: rows behind lens (all ones from the start),
    later new tokens (causal), rows before the window."""
    L, window = 300, 150
    c = Case(kind, 2, 1, 128, 16, [L, L], [new, new])
    c.fill()
    k, v = c.rand(2 * new, 1, 128), c.rand(2 * new, 1, 128)
    bad = torch.zeros(2 * new, dtype=torch.bool)
    # the last two tokens of the first sequence
    bad[new - 1] = bad[new - 2] = True
    k[new - 1], v[new - 1], v[new - 2] = math.nan, math.inf, math.nan
    c.ctx.append(0, None, k, v, c.lens, c.table, starts=c.starts)
    # rows before any window of the second sequence
    head = L - new + 1 - window
    first = torch.tensor([0, head], dtype=torch.int32, device="cuda")
    junk = torch.full((head, 1, 128), math.inf, dtype=k.dtype, device="cuda")
    c.ctx.append(0, None, junk, junk, first, c.table, starts=torch.tensor([0, 0, head], dtype=torch.int32, device="cuda"))
    q = c.rand(2 * new, 2, 128)
    out = torch.zeros(2 * new, 2, 128, dtype=TORCH[c.out], device="cuda")
    lse = torch.zeros(2 * new, 2, device="cuda")
    c.ctx.attend(0, q, c.lens, c.table, out, starts=c.starts, max_new=new, window=window, lse=lse)
    c.ctx.status_sync()
    assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all()
    K, V = R.cache_values(c.pages, kind, 0, 128, 16)
    KS, VS = R.cache_sizes(c.pages, kind, 0, 128, 16)
    rd = roundings(kind, c.out, 2 * new)
    for b in range(2):
        k64, v64, ks, vs = (R.rows_of(x, c.table[b], L, 16) for x in (K, V, KS, VS))
        ref, rl, ma, sa = R.attend(q[b * new:(b + 1) * new].double(), k64, v64, L - new, window, sizes=(ks, vs))
        good = ~bad[b * new:(b + 1) * new].cuda()
        bound = R.out_bound(ref, ma, sa, 128, L, HALF[c.out], **rd)
        assert ((out[b * new:(b + 1) * new].double() - ref).abs() <= bound)[good].all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, INT4])
@pytest.mark.parametrize("new", [1, 40])
def test_sharp_and_flat_attention(kind, new):
    """Keys of one direction with a strongly varying length (logits from -600 to 600), and all-equal logits."""
    c = Case(kind, 4, 2, 128, 16, [400, 37], [new, new])
    total = 437
    u = torch.nn.functional.normalize(c.rand(1, 2, 128, dtype=torch.float32), dim=-1)
    size = c.rand(total, 1, 1, dtype=torch.float32) * 100
    k, v = (u * size).to(TORCH[c.io]), c.rand(total, 2, 128)
    c.ctx.append(0, None, k, v, c.lens, c.table, starts=torch.tensor([0, 400, 437], dtype=torch.int32, device="cuda"))
    q = (u.repeat_interleave(2, 1) * 20).to(TORCH[c.io]).repeat(2 * new, 1, 1)
    c.check_attend(q=q, **roundings(kind, c.out, 2 * new))
    out, lse = c.check_attend(q=q * 0, **roundings(kind, c.out, 2 * new))


@pytest.mark.gpu
@pytest.mark.parametrize("scales", [(1e-4, 1e-4), (1.0, 1e-30), (1.0, 1e30), (1e-20, 1e-20)])
def test_int4_values_of_any_size(scales):
    """4-bit rows whose values change in size from token to token, far outside fp16's range."""
    c = Case(INT4, 4, 2, 128, 16, [200, 90], out=F32)
    n = 290
    size = torch.logspace(math.log10(scales[0]), math.log10(scales[1]), n, device="cuda")[torch.randperm(n, generator=c.gen, device="cuda")]
    k = c.rand(n, 2, 128) * 0.1
    v = (c.rand(n, 2, 128, dtype=torch.float32) * size[:, None, None]).to(TORCH[c.io])
    c.ctx.append(0, None, k, v, c.lens, c.table, starts=torch.tensor([0, 200, 290], dtype=torch.int32, device="cuda"))
    for amp in (1.0, 1e-6, 300.0):
        q = (c.rand(2, 4, 128, dtype=torch.float32) * amp).to(TORCH[c.io])
        c.check_attend(q=q, **roundings(INT4, F32, 2))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, INT4, F32])
def test_scale_strides_and_padded_table(kind):
    """A scale of the caller's, queries as a slice, a table with longer rows than the batch uses."""
    c = Case(kind, 6, 2, 128, 32, [70, 5, 300], max_batch=50)
    c.fill()
    buf = c.rand(3, 10, 128)
    wide = torch.full((3, c.per + 9), -1, dtype=torch.int32, device="cuda")
    wide[:, : c.per] = c.table
    c.check_attend(q=buf[:, 2:8], scale=0.31, table=wide[:, : c.per + 1], **roundings(kind, c.out, 3))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, INT4])
def test_sequences_share_pages(kind):
    c = Case(kind, 4, 1, 128, 16, [160, 170, 165], extra_pages=0)
    c.table_h[1, :9] = c.table_h[0, :9]
    c.table_h[2, :10] = c.table_h[0, :10]
    c.table = c.table_h.cuda()
    c.fill()   # equal rows are written three times with different values: whichever stays is read by all
    c.check_attend(**roundings(kind, c.out, 4))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, INT4, F32])
@pytest.mark.parametrize("new", [1, 70])
def test_pages_far_into_a_large_cache(kind, new):
    """Offsets beyond 2^32 bytes: the sequences' pages are the last of a cache of more than 4 GB."""
    d, hk, page = 128, 2, 64
    size = mkv.paged_page_bytes(hk, d, page, kind)
    n_pages = (1 << 32) // size + 40
    c = Case(kind, 4, hk, d, page, [200, 129], [new, new], extra_pages=n_pages)
    top = c.pages.shape[1] - 1
    for b in range(2):
        for i in range(c.per):
            if c.table_h[b, i] >= 0:
                c.table_h[b, i] = top
                top -= 1
    c.table = c.table_h.cuda()
    c.fill()
    assert (c.pages[0, : top + 1].view(torch.uint8)[:: 4099] == 255).all()
    low = int(c.table_h[c.table_h >= 0].min())
    # compare against the used pages alone
    whole, c.pages = c.pages, c.pages[:, low:].contiguous()
    table = c.table.clone()
    c.table_h = torch.where(c.table_h >= 0, c.table_h - low, c.table_h)
    c.check_attend(table=table, **roundings(kind, c.out, 2 * new))
    del whole


@pytest.mark.gpu
def test_what_the_kernels_find_wrong_is_a_status():
    for kind in (BF16, INT4, F32):
        for bad in ("page", "negative", "long", "starts"):
            c = Case(kind, 2, 1, 128, 16, [40, 20], [2, 2])
            c.fill()
            before = c.pages.clone()
            k, q = c.rand(4, 1, 128), c.rand(4, 2, 128)
            out = torch.zeros(4, 2, 128, dtype=TORCH[c.out], device="cuda")
            code = 1
            if bad == "page":
                c.table[0, 2] = c.pages.shape[1]
            elif bad == "negative":
                c.table[0, 2] = -1
            elif bad == "long":
                c.lens[0] = c.per * 16 + 2
                code = 3
            else:
                c.starts[1] = 9
            c.ctx.append(0, None, k, k, c.lens, c.table, starts=c.starts)
            with pytest.raises(mkv.MkvError) as e:
                c.ctx.status_sync()
            assert e.value.code == code
            c.ctx.reset()
            c.ctx.status_sync()
            # nothing but the second sequence's two rows was written
            same = (before.view(torch.uint8) == c.pages.view(torch.uint8)).flatten(1)
            assert int((~same).sum()) <= 2 * 2 * 128 * 4
            c.ctx.attend(0, q, c.lens, c.table, out, starts=c.starts, max_new=2)
            with pytest.raises(mkv.MkvError) as e:
                c.ctx.status_sync()
            assert e.value.code == code
            c.ctx.reset()
    # more new tokens than promised
    c = Case(BF16, 2, 1, 128, 16, [40, 20], [3, 2])
    c.fill()
    q = c.rand(5, 2, 128)
    c.ctx.attend(0, q, c.lens, c.table, torch.zeros_like(q), starts=c.starts, max_new=2)
    with pytest.raises(mkv.MkvError) as e:
        c.ctx.status_sync()
    assert e.value.code == 3


@pytest.mark.gpu
def test_refusals_of_the_calls():
    """Checked on the host, before anything is enqueued."""
    c = Case(BF16, 4, 2, 128, 16, [5, 6])
    L, h = c.ctx._L, c.ctx._ctx
    n0 = c.ctx.launch_count()
    buf = torch.zeros(1 << 16, dtype=torch.bfloat16, device="cuda")
    p, ln, tb = buf.data_ptr(), c.lens.data_ptr(), c.table.data_ptr()

    def app(**kw):
        a = dict(layer=0, q=p, qs=512, k=p, ks=256, v=p, vs=256, qo=p, n=2, b=2, st=None, ln=ln, tb=tb, ts=c.per)
        a.update(kw)
        return L.mkv_paged_append(h, a["layer"], a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["qo"], a["n"], a["b"],
                                  a["st"], a["ln"], a["tb"], a["ts"], None, None)

    for kw in [dict(layer=1), dict(layer=-1), dict(n=-1), dict(b=-1), dict(n=3), dict(k=None), dict(v=None), dict(qo=None),
               dict(q=None), dict(qs=511), dict(ks=255), dict(vs=260), dict(k=p + 2), dict(qo=p + 8), dict(ln=None),
               dict(tb=None), dict(ts=0), dict(ln=ln + 2), dict(tb=tb + 1), dict(st=p + 2)]:
        assert app(**kw) == 1, kw
    assert app(n=3, b=3) == 3 and app(ts=1 << 27) == 5
    assert app(n=0, b=0) == 0

    def att(**kw):
        a = dict(layer=0, q=p, qs=512, out=p, lse=None, n=2, b=2, st=None, mn=1, ln=ln, tb=tb, ts=c.per, sc=0.0, w=0)
        a.update(kw)
        return L.mkv_paged_attend(h, a["layer"], a["q"], a["qs"], a["out"], a["lse"], a["n"], a["b"], a["st"], a["mn"], a["ln"],
                                  a["tb"], a["ts"], a["sc"], a["w"], None)

    for kw in [dict(layer=1), dict(q=None), dict(out=None), dict(out=p + 4), dict(qs=500), dict(mn=0), dict(w=-1), dict(sc=-1.0),
               dict(sc=math.nan), dict(sc=math.inf), dict(n=1), dict(lse=p + 2)]:
        assert att(**kw) == 1, kw
    assert att(n=3, b=3) == 3

    def rd(**kw):
        a = dict(layer=0, b=2, first=None, ln=ln, tb=tb, ts=c.per, K=p, V=p, rows=4)
        a.update(kw)
        return L.mkv_paged_read(h, a["layer"], a["b"], a["first"], a["ln"], a["tb"], a["ts"], a["K"], a["V"], a["rows"], None)

    for kw in [dict(layer=2), dict(rows=-1), dict(K=None), dict(V=p + 4), dict(ln=None), dict(first=p + 2)]:
        assert rd(**kw) == 1, kw
    assert rd(rows=0) == 0 and rd(b=3) == 3
    f = (C.c_float * 64)()
    assert L.mkv_paged_set_rotation(h, f, 24, 0) == 5 and L.mkv_paged_set_rotation(h, f, 144, 0) == 1
    assert L.mkv_paged_set_rotation(h, None, 16, 0) == 1 and L.mkv_paged_set_rotation(h, f, 16, 2) == 1
    assert c.ctx.launch_count() == n0
    # the binding
    q, k = c.rand(2, 4, 128), c.rand(2, 2, 128)
    with pytest.raises(ValueError):
        c.ctx.attend(0, q.float(), c.lens, c.table, q)
    with pytest.raises(ValueError):
        c.ctx.attend(0, q.transpose(1, 2).contiguous().transpose(1, 2), c.lens, c.table, q)
    with pytest.raises(ValueError):
        c.ctx.attend(0, q, c.lens.long(), c.table, q)
    with pytest.raises(ValueError):
        c.ctx.append(0, q, k, k[:1], c.lens, c.table, q_out=q)
    with pytest.raises(ValueError):
        c.ctx.attend(0, q[:1], c.lens, c.table, q[:1])
    with pytest.raises(ValueError):
        c.ctx.attend(0, q.cpu(), c.lens, c.table, q)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, F32, INT4])
def test_steps_together_and_on_into_a_context(kind):
    """As they are used: a prompt appended in pieces and attended as it grows, single tokens decoded, then the
    cache read into the prompt pool of a Moment-KV context, whose attention agrees with the cache's."""
    hq, hk, d = (4, 1, 64) if kind == F32 else (8, 2, 128)
    io = F32 if kind == F32 else BF16
    c = Case(kind, hq, hk, d, 16, [120, 120], [0, 0], out=F32, extra_pages=0)
    inv = (10000.0 ** (-np.arange(0, d, 2) / d)).astype(np.float32)
    c.ctx.set_rotation(inv)
    have = [0, 0]
    for new in ([37, 20], [1, 0], [40, 61], [1, 1], [1, 1], [3, 5]):
        have = [a + n for a, n in zip(have, new)]
        c.lens_h, c.new_h, c.T = have, new, sum(new)
        c.starts_h = [0, new[0], sum(new)]
        c.starts = torch.tensor(c.starts_h, dtype=torch.int32, device="cuda")
        c.lens = torch.tensor(have, dtype=torch.int32, device="cuda")
        q, k, v = c.rand(c.T, hq, d), c.rand(c.T, hk, d), c.rand(c.T, hk, d)
        turned = torch.zeros_like(q)
        c.ctx.append(0, q, k, v, c.lens, c.table, q_out=turned, starts=c.starts)
        c.check_attend(q=turned, **roundings(kind, F32, hq // hk * max(new)))
    n = max(have)
    K = torch.zeros(2, hk, n, d, dtype=TORCH[io], device="cuda")
    V = torch.zeros_like(K)
    c.ctx.read(0, c.lens, c.table, K, V)
    m = mkv.MomentKV(1, hq, hk, d, 8, 0.9, 2, n, kv_dtype=io, out_dtype=F32)
    m.prefill(0, K, V, have)
    q = c.rand(2, hq, d)
    got, want = torch.zeros(2, hq, d, device="cuda"), torch.zeros(2, hq, d, device="cuda")
    m.attend_only(0, q, want)
    m.status_sync()
    c.ctx.attend(0, q, c.lens, c.table, got)
    c.ctx.status_sync()
    # the rows handed on are rounded to bf16 where the cache holds 4 bits
    assert (got - want).abs().max() <= want.abs().max() * (2.0 ** -6 if kind == INT4 else 2.0 ** -14)
    m.close()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, INT4, F32])
@pytest.mark.parametrize("new", [1, 3, 80])
def test_captured_replayed_and_on_other_streams(kind, new):
    """A recorded append + attend, replayed after the inputs, lengths and pages changed; a padded batch; the
    same bits on another stream, and from a second handle at the same time."""
    c = Case(kind, 4, 2, 128, 16, [200, 150, 90], [new, new, new])
    c.fill()
    q, k, v = c.rand(3 * new, 4, 128), c.rand(3 * new, 2, 128), c.rand(3 * new, 2, 128)
    out, qo = torch.full_like(q, 7.0), torch.zeros_like(q)
    rd = roundings(kind, c.out, 2 * new)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.ctx.append(0, q, k, v, c.lens, c.table, q_out=qo, starts=c.starts)
        c.ctx.attend(0, qo, c.lens, c.table, out, starts=c.starts, max_new=new)
    torch.cuda.synchronize()
    c.compare(qo, out, None, **rd)
    once = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.ctx.append(0, q, k, v, c.lens, c.table, q_out=qo, starts=c.starts)
        c.ctx.attend(0, qo, c.lens, c.table, out, starts=c.starts, max_new=new)
    out.fill_(7)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, once)
    # shorter sequences, the last one gone (its rows belong to none), other values
    c.lens_h = [140, 97, 0]
    c.lens.copy_(torch.tensor(c.lens_h, dtype=torch.int32))
    c.starts_h = [0, new, 2 * new, 2 * new]
    c.starts.copy_(torch.tensor(c.starts_h, dtype=torch.int32))
    for t in (q, k, v):
        t.copy_(c.rand(*t.shape))
    out.fill_(7)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    c.ctx.status_sync()
    c.T = 3 * new
    c.compare(qo, out, None, **rd)
    first = out.clone()
    # two handles over the same pages at the same time
    other = mkv.PagedKV(c.pages, 4, 2, 128, 16, 3, kv_dtype=kind, io_dtype=c.io, out_dtype=c.out)
    outs = [torch.full_like(out, 7.0) for _ in range(16)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for i, o in enumerate(outs):
        (c.ctx, other)[i % 2].attend(0, qo, c.lens, c.table, o, starts=c.starts, max_new=new, stream=streams[i % 2])
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, first)
    other.close()


@pytest.mark.gpu
def test_empty_batches():
    c = Case(BF16, 4, 2, 128, 16, [0, 0], max_batch=4)
    e = torch.zeros(0, 4, 128, dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros(0, 2, 128, dtype=torch.bfloat16, device="cuda")
    none, tab = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, 1, dtype=torch.int32, device="cuda")
    c.ctx.append(0, e, kv, kv, none, tab, q_out=e.clone())
    c.ctx.attend(0, e, none, tab, e.clone())
    st = torch.zeros(3, dtype=torch.int32, device="cuda")
    c.ctx.append(0, e, kv, kv, c.lens, c.table, q_out=e.clone(), starts=st)
    c.ctx.attend(0, e, c.lens, c.table, e.clone(), starts=st)
    # rows that belong to no sequence
    q = c.rand(5, 4, 128)
    out = torch.full_like(q, 7.0)
    c.ctx.attend(0, q, c.lens, c.table, out, starts=st, max_new=5)
    c.ctx.status_sync()
    assert (out == 7).all()
    # sequences without tokens, one query each: zeros
    out = torch.full((2, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(2, 4, device="cuda")
    c.ctx.attend(0, q[:2], c.lens, c.table, out, lse=lse)
    c.ctx.status_sync()
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, INT4])
def test_large_batches_and_long_sequences(kind):
    """More sequences than the grid has blocks, and one sequence that all blocks share."""
    lens = [(i * 37) % 90 for i in range(1500)]
    c = Case(kind, 4, 1, 128, 16, lens, seed=5)
    c.fill()
    c.check_attend(**roundings(kind, c.out, 4))
    c = Case(kind, 8, 1, 128, 64, [70001], out=F32, seed=6)
    c.fill()
    a, _ = c.check_attend(q=c.rand(1, 8, 128) * 4, **roundings(kind, F32, 8))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, INT4])
@pytest.mark.parametrize("window", [0, 1500])
def test_long_pieces(kind, window):
    """Many tiles and several units for every block of the grid, units cut between blocks: against the plain form on
    sampled tokens, and the same bits again."""
    c = Case(kind, 8, 2, 128, 64, [2900, 4111, 700, 3333], [350, 1, 700, 97], out=F32, seed=11)
    c.fill()
    q = c.rand(c.T, 8, 128) * 3
    outs = []
    for _ in range(3):
        out = torch.zeros(c.T, 8, 128, device="cuda")
        lse = torch.zeros(c.T, 8, device="cuda")
        c.ctx.attend(0, q, c.lens, c.table, out, starts=c.starts, max_new=700, window=window, lse=lse)
        outs.append((out, lse))
    c.ctx.status_sync()
    assert all(torch.equal(a, outs[0][0]) and torch.equal(b, outs[0][1]) for a, b in outs[1:])
    K, V = R.cache_values(c.pages, kind, 0, 128, 64)
    KS, VS = R.cache_sizes(c.pages, kind, 0, 128, 64)
    rd = roundings(kind, F32, 2800)
    for b, (a, e) in enumerate(zip(c.starts_h, c.starts_h[1:])):
        k, v, ks, vs = (R.rows_of(x, c.table[b], c.lens_h[b], 64) for x in (K, V, KS, VS))
        for i in sorted({a, (2 * a + e) // 3, (a + e) // 2, max(a, e - 2), e - 1}):
            ref, lse, ma, sa = R.attend(q[i:i + 1].double(), k, v, c.lens_h[b] - (e - i), window, sizes=(ks, vs))
            bound = R.out_bound(ref, ma, sa, 128, c.lens_h[b], HALF[F32], **rd)
            assert ((outs[0][0][i].double() - ref[0]).abs() <= bound[0]).all(), (b, i)
            err = (outs[0][1][i].double() - lse[0]).abs()
            assert (err <= R.lse_bound(lse, sa, 128, c.lens_h[b], rd["e_p"], rd.get("e_k", 0.0))[0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, INT4, F32])
@pytest.mark.parametrize("new", [6, 7, 16, 17, 24, 25])
def test_either_side_of_the_choice_of_a_kernel(kind, new):
    """24 and 28, 64 and 68, 96 and 100 rows of a sequence and head, in a batch that fills the GPU and in a small one."""
    for batch in (40, 2):
        lens = [new + (37 * i) % 150 for i in range(batch)]
        c = Case(kind, 8, 2, 64, 16, lens, [new if i % 3 else 1 + i % new for i in range(batch)], seed=new)
        c.fill()
        c.check_attend(max_new=new, **roundings(kind, c.out, 4 * new))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [BF16, INT4, F32])
def test_windows_of_any_size(kind):
    c = Case(kind, 4, 2, 128, 16, [300, 40], [130, 40])
    c.fill()
    q = c.rand(170, 4, 128)
    whole, _ = c.check_attend(q=q, **roundings(kind, c.out, 260))
    for w in (300, 1 << 29, (1 << 30) - 1, 1 << 30, (1 << 31) - 1):
        out, _ = c.check_attend(q=q, window=w, **roundings(kind, c.out, 260))
        assert torch.equal(out, whole)
