"""The 8-bit KV cache's operators (include/ebrl_kv8.h) against a plain float64
form: what a write stores, byte for byte, and attention within bounds that
follow from its arithmetic; the calls that are refused."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_27547_amd import ebrl as E
from tests import kv8_ref as R

gpu = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------ no GPU needed --

def _attn_args(**kw):
    a = E.Kv8AttnArgs(dtype=E.DTYPE_BF16, n=2, rows=2, max_q_len=1, max_kv_len=100, q_heads=4, causal=1, scale=0.125,
                      ldq=256, ldo=256)
    for f in ("q", "out", "row_start", "kv_len"):
        setattr(a, f, 4096 * (1 + "q out row_start kv_len".split().index(f)))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _cache(**kw):
    c = E.Kv8Cache(1 << 20, 2 << 20, 3 << 20, 8, 2, 4, 2, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _attn(c, a):
    return E.lib().ebrl_op_kv8_attn(ctypes.byref(c), ctypes.byref(a), None)


@pytest.mark.parametrize("bad", [
    dict(codes=0), dict(codes=(1 << 20) + 8), dict(scales=0), dict(block_table=0), dict(num_blocks=0), dict(table_rows=0),
    dict(table_stride=0), dict(table_stride=1 << 27), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=32),
    dict(head_dim=96)])
def test_attn_refuses_cache(bad):
    assert _attn(_cache(**bad), _attn_args()) == -1


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(n=-1), dict(rows=-1), dict(max_q_len=-1), dict(max_kv_len=-1), dict(max_kv_len=(1 << 30) + 1),
    dict(q_heads=0), dict(q_heads=5), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(scale=3e38), dict(q=0), dict(out=0), dict(q=4096 + 8), dict(ldq=255), dict(ldq=260), dict(ldo=128),
    dict(row_start=0), dict(kv_len=0), dict(out=4096), dict(max_kv_len=10000)])   # the last: needs a workspace
def test_attn_refuses_arguments(bad):
    assert _attn(_cache(), _attn_args(**bad)) == -1


def test_attn_of_nothing_is_ok():
    for kw in (dict(n=0), dict(rows=0), dict(max_q_len=0)):
        assert _attn(_cache(), _attn_args(**kw)) == 0


def _write_args(**kw):
    a = E.Kv8WriteArgs(dtype=E.DTYPE_BF16, n=2, rows=4, max_len=3, q_heads=4, n_axes=2, tab_rows=10, ldq=256, ldk=128,
                       ldv=128, ldq_out=256)
    a.sections[0], a.sections[1] = 20, 12
    for i, f in enumerate(("q", "k", "v", "q_out", "row_start", "pos0", "axis_pos", "cos_tab", "sin_tab")):
        setattr(a, f, 4096 * (1 + i))
    for k, v in kw.items():
        if k == "sections":
            for i, x in enumerate(v):
                a.sections[i] = x
        else:
            setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad", [
    dict(dtype=7), dict(n=-1), dict(rows=-1), dict(max_len=-1), dict(q_heads=-1), dict(n_axes=4), dict(n_axes=-1),
    dict(n_axes=0), dict(sections=(20, 13)), dict(sections=(32, 0)), dict(sections=(33, -1)), dict(tab_rows=0),
    dict(cos_tab=0), dict(sin_tab=4), dict(axis_pos=0), dict(k=0), dict(v=4104), dict(ldk=127), dict(ldv=130),
    dict(q=0), dict(q_out=0), dict(ldq_out=8), dict(row_start=0), dict(pos0=0), dict(q_out=4096, ldq_out=512)])
def test_write_refuses_arguments(bad):
    assert E.lib().ebrl_op_kv8_write(ctypes.byref(_cache()), ctypes.byref(_write_args(**bad)), None) == -1


@pytest.mark.parametrize("bad", [dict(codes=0), dict(codes=8), dict(scales=0), dict(block_table=0), dict(head_dim=80),
                                 dict(num_blocks=-1)])
def test_write_refuses_cache(bad):
    assert E.lib().ebrl_op_kv8_write(ctypes.byref(_cache(**bad)), ctypes.byref(_write_args()), None) == -1


def test_write_of_nothing_is_ok():
    for kw in (dict(n=0), dict(rows=0), dict(max_len=0)):
        assert E.lib().ebrl_op_kv8_write(ctypes.byref(_cache()), ctypes.byref(_write_args(**kw)), None) == 0


def test_workspace_sizes():
    c = _cache(table_stride=10000)

    def need(**kw):
        return E.lib().ebrl_op_kv8_attn_workspace(ctypes.byref(c), ctypes.byref(_attn_args(**kw)))
    assert need(max_kv_len=1) == 0 and need(n=0, max_kv_len=100000) == 0
    assert need(max_kv_len=100000) > 0
    assert need(q_heads=3) == -1 and need(dtype=5) == -1
    # enough sequences fill the chip without cutting their keys
    assert need(n=4096, rows=4096, max_kv_len=4096) == 0


def test_binding_refuses():
    codes, scales = E.kv8_alloc(4, 2, 64, device="cpu")
    table = torch.zeros((1, 4), dtype=torch.int32)
    k = torch.zeros((1, 128), dtype=torch.bfloat16)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    ok = dict(codes=codes, scales=scales, block_table=table, k=k, v=k, row_start=i32(0, 1), pos0=i32(0), max_len=1)

    def refused(f, **kw):
        with pytest.raises(E.EbrlError):
            f(**kw)
    refused(E.op_kv8_write, **ok)                                             # not on a GPU
    for bad in (dict(codes=codes.view(torch.uint8)[:, :1]), dict(codes=codes.float()), dict(scales=scales.double()),
                dict(block_table=table.long()), dict(v=k.float()), dict(k=k[:, :64]), dict(pos0=i32(0).long()),
                dict(row_start=i32(0)), dict(q=k), dict(k=torch.zeros((1, 128), dtype=torch.float16)),
                dict(sections=(32,)), dict(sections=(8, 8, 8, 8)), dict(max_len=-1), dict(max_len=1 << 32)):
        refused(E.op_kv8_write, **{**ok, **bad})
    at = dict(codes=codes, scales=scales, block_table=table, q=k, out=k.clone(), row_start=i32(0, 1), kv_len=i32(1),
              max_q_len=1, max_kv_len=1)
    for bad in (dict(), dict(out=k.float()), dict(q=k[:, :65], out=k[:, :65]), dict(kv_len=i32(1, 1)),
                dict(q=k.half(), out=k.half()), dict(stream=0), dict(out=k[:, :64]), dict(max_kv_len=1 << 32),
                dict(max_q_len=-1), dict(q=k[0], out=k[0])):
        refused(E.op_kv8_attn, **{**at, **bad})


def test_binding_refuses_what_the_structs_do_not_hold():
    codes, scales = E.kv8_alloc(4, 2, 64, device="cpu")
    table = torch.zeros((1, 4), dtype=torch.int32)
    k = torch.zeros((1, 128), dtype=torch.bfloat16)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    tab = torch.zeros(4, 32)
    write = dict(codes=codes, scales=scales, block_table=table, k=k, v=k, row_start=i32(0, 1), pos0=i32(0), max_len=1,
                 cos=tab, sin=tab)
    for bad in (dict(sections=(1 << 31,)), dict(sections=(31.5,)), dict(codes=codes[:, :, 0]), dict(codes=codes[..., :0])):
        with pytest.raises(E.EbrlError):
            E.op_kv8_write(**{**write, **bad})
    attn = dict(codes=codes, scales=scales, block_table=table, q=k, out=k.clone(), row_start=i32(0, 1), kv_len=i32(1),
                max_q_len=1, max_kv_len=1, workspace=torch.empty(0, dtype=torch.uint8))
    for bad in (dict(scale=1e39), dict(codes=codes[..., :0]), dict(block_table=table[0])):
        with pytest.raises(E.EbrlError):
            E.op_kv8_attn(**{**attn, **bad})
    sizes = dict(codes=codes, block_table=table, q=k, n=1, max_q_len=1, max_kv_len=1)
    assert E.kv8_attn_workspace(**sizes).numel() == 0
    for bad in (dict(n=-1), dict(n=1 << 31), dict(codes=codes[0]), dict(codes=codes[..., :0]), dict(block_table=table[0]),
                dict(q=k[0]), dict(max_kv_len=1 << 31)):
        with pytest.raises(E.EbrlError):
            E.kv8_attn_workspace(**{**sizes, **bad})


def test_packed_structs_are_the_c_structs():
    for packed, struct in ((E._KV8_CACHE, E.Kv8Cache), (E._KV8_WRITE, E.Kv8WriteArgs), (E._KV8_ATTN, E.Kv8AttnArgs)):
        values = list(range(1, 1 + len(packed.unpack(bytes(packed.size)))))
        a = struct.from_buffer_copy(packed.pack(*values))
        got = []
        for name, _ in struct._fields_:
            x = getattr(a, name)
            got += list(x) if name == "sections" else [x]
        assert packed.size == ctypes.sizeof(struct) and got == values


def test_reference_encode_matches_torch():
    """The test's own e4m3 rounding against torch's, ties and small values among them."""
    x = np.concatenate([np.linspace(-448, 448, 4001), R.CODE[:127], (R.CODE[:126] + R.CODE[1:127]) / 2,
                        np.random.default_rng(0).standard_normal(4000) * 2.0 ** -7])
    x = x.astype(np.float32)
    t = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(t, R.encode(x))


# ------------------------------------------------------------------ the GPU --

def _bits(t):
    return t.view(torch.uint8).cpu().numpy()


class Pool:
    """A cache whose sequences hold `lens` tokens of random values, pages in random order."""

    def __init__(self, seed, lens, hkv, hd, room=0, extra=3, spread=1.0):
        self.rng = np.random.default_rng(seed)
        self.hkv, self.hd = hkv, hd
        pages = [(n + room + R.PAGE - 1) // R.PAGE for n in lens]
        self.nb = sum(pages) + extra
        order = self.rng.permutation(self.nb).astype(np.int32)
        self.table = np.full((len(lens), max(pages + [1]) + 1), -1, np.int32)
        at = 0
        for i, p in enumerate(pages):
            self.table[i, :p] = order[at:at + p]
            at += p
        # slots that hold no token are NaN codes, and so is what pages without any hold
        self.codes = np.full((self.nb, 2, hkv, R.PAGE * hd), 0x7F, np.uint8)
        self.scales = np.full((self.nb, 2, hkv), np.nan, np.float32)
        for i, n in enumerate(lens):
            if n:
                x = self.rng.standard_normal((2, n, hkv, hd)) * np.exp2(self.rng.uniform(-spread, spread, (2, n, 1, 1)))
                R.write(self.codes, self.scales, self.table[i:i + 1], x[0], x[1], [0, n], [0], n)

    def gpu(self):
        codes = torch.from_numpy(self.codes.copy()).cuda().view(torch.float8_e4m3fn)
        return codes, torch.from_numpy(self.scales.copy()).cuda(), torch.from_numpy(self.table).cuda()


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def _tables(n, hd):
    ang = np.arange(n)[:, None] * 10000.0 ** (-2.0 * np.arange(hd // 2) / hd)
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def _rows(rng, rows, heads, hd, dt, pad=0):
    """(device rows, strided if pad, and their float64 values)"""
    t = torch.from_numpy(rng.standard_normal((rows, heads * hd + pad))).to(dt).cuda()[:, :heads * hd]
    return t, t.double().cpu().numpy().reshape(rows, heads, hd)


def _same_codes(got, want):
    """Codes equal; a zero's sign and a NaN's may differ."""
    g, w = R.CODE[got], R.CODE[want]
    np.testing.assert_array_equal(g, w)


def _check_write(pool, dt, hq, past, new, sections, pad, seed, max_len=None, seq=None, outside=2):
    rng = np.random.default_rng(seed)
    hkv, hd = pool.hkv, pool.hd
    rows = sum(new) + outside
    start = np.concatenate([[0], np.cumsum(new)])
    k, k64 = _rows(rng, rows, hkv, hd, dt, pad)
    v, v64 = _rows(rng, rows, hkv, hd, dt, 2 * pad)
    q, q64 = _rows(rng, rows, hq, hd, dt, pad)
    cos, sin = _tables(200, hd)
    axes = len(sections)
    axis_pos = rng.integers(0, 200, (rows, axes)).astype(np.int32) if axes > 1 else None
    codes, scales, table = pool.gpu()
    q_out = torch.full_like(q, 7.0)
    mx = max(list(new) + [1]) if max_len is None else max_len
    E.op_kv8_write(codes, scales, table, k, v, _ints(start), _ints(past), mx, q=q if axes else None,
                   q_out=q_out if axes else None, sections=sections,
                   axis_pos=None if axis_pos is None else torch.from_numpy(axis_pos).cuda(),
                   cos=torch.from_numpy(cos).cuda() if axes else None, sin=torch.from_numpy(sin).cuda() if axes else None,
                   seq=None if seq is None else _ints(seq))
    wc, ws = pool.codes.copy(), pool.scales.copy()
    wq = R.write(wc, ws, pool.table, k64, v64, list(start), list(past), mx, list(sections), axis_pos, cos, sin, seq,
                 q64 if axes else None)
    _same_codes(_bits(codes), wc)
    np.testing.assert_array_equal(scales.cpu().numpy(), ws)
    if axes:
        got = q_out.double().cpu().numpy().reshape(wq.shape)
        out = np.isnan(wq)
        assert np.all(got[out] == 7.0)
        half = torch.finfo(dt).eps / 2
        assert np.all(np.abs(got - wq)[~out] <= half * np.abs(wq[~out]) * (1 + 2.0 ** -20) + 1e-38)
    return codes, scales


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 4, 64), (6, 2, 128), (8, 8, 128), (5, 1, 64)])
@pytest.mark.parametrize("past,new", [([0], [1]), ([0, 0], [16, 33]), ([5, 15, 16, 31], [1, 1, 1, 1]),
                                      ([3, 0, 17, 40], [20, 0, 60, 7])])
def test_write_one_axis(dtype, hq, hkv, hd, past, new):
    pool = Pool(1, past, hkv, hd, room=max(new) + 1)
    _check_write(pool, DT[dtype], hq, past, new, (hd // 2,), 0, 2)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,sections", [(64, ()), (64, (16, 16)), (64, (1, 30, 1)), (128, (32, 16, 16)), (128, (33, 31)),
                                         (128, (2, 61, 1)), (128, ())])
def test_write_axes_and_strides(dtype, hd, sections):
    past, new = [9, 0, 32, 2], [40, 17, 1, 14]
    pool = Pool(3, past, 3, hd, room=41)
    _check_write(pool, DT[dtype], 6, past, new, sections, 8, 4)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,sections", [(64, (32,)), (64, (3, 28, 1)), (128, ()), (128, (64,)), (128, (32, 16, 16)),
                                         (128, (30, 34))])
@pytest.mark.parametrize("hq,hkv", [(9, 3), (17, 1), (24, 12)])
def test_write_one_token(dtype, hd, sections, hq, hkv):
    """A token a sequence, in every slot of a page, before a page that is not there too."""
    past = list(range(18)) + [31, 47, 60]
    pool = Pool(50, past, hkv, hd, room=3)
    pool.table[4, 0], pool.table[20, 3] = -1, pool.nb
    _check_write(pool, DT[dtype], hq, past, [1] * len(past), sections, 8, 51)
    _check_write(pool, DT[dtype], hq, past, [1, 0] * 10 + [2], sections, 0, 52, max_len=1)


@gpu
def test_write_many_heads_and_pages():
    """Enough (page, head) pairs for the waves to take several heads in turn."""
    past, new = list(range(0, 120, 3)), [50] * 40
    pool = Pool(5, past, 40, 64, room=51)
    _check_write(pool, torch.bfloat16, 41, past, new, (20, 12), 0, 6)


@gpu
def test_write_keeps_to_its_bounds():
    """Row ranges past the rows and max_len are cut, unknown table rows and
    pages that are none are skipped, positions are cut to the tables."""
    past = [4, 18, 0, 30]
    pool = Pool(7, past, 2, 64, room=40)
    pool.table[1, 2] = pool.nb                    # a page past the pool ...
    pool.table[3, 2] = -5                         # ... and one before it
    _check_write(pool, torch.bfloat16, 2, past, [20, 30, 6, 25], (32,), 0, 8, max_len=19)
    _check_write(pool, torch.bfloat16, 2, past, [20, 30, 6, 25], (32,), 0, 9, seq=[0, -1, 4, 3])
    # rows that end in the middle of the last sequence, a position past the table's row
    _check_write(pool, torch.bfloat16, 2, [4, 18, 0, pool.table.shape[1] * 16 - 3], [3, 3, 3, 9], (32,), 0, 10, outside=-4)
    _check_write(pool, torch.bfloat16, 2, [-1, 1 << 30, 0, 190], [3, 3, 3, 9], (32,), 0, 11)


LEAST, MOST = -2 ** 31, 2 ** 31 - 1


@gpu
@pytest.mark.parametrize("max_len", [1, 40])
def test_write_of_any_numbers(max_len):
    """Device data that says anything: nothing out of bounds is touched, what is in bounds is written."""
    rng = np.random.default_rng(70)
    past = [4, 18, 0, 30, 7, 2]
    pool = Pool(71, past, 2, 64, room=60)
    pool.table[4] = [LEAST, MOST, -1, pool.nb, pool.nb - 1, 0][:pool.table.shape[1]] + [0] * max(0, pool.table.shape[1] - 6)
    n, rows = 9, 50
    k, k64 = _rows(rng, rows, 2, 64, torch.bfloat16)
    q, q64 = _rows(rng, rows, 2, 64, torch.bfloat16)
    axis = rng.choice([LEAST, -1, 0, 3, 199, 200, MOST], (rows, 2)).astype(np.int32)
    cos, sin = _tables(200, 64)
    # each sequence's rows are its own: the numbers that are no bounds come between
    start = [5, 9, LEAST, 3, 17, MOST, 20, -4, 40, 2 ** 30]
    pos0 = [4, 18, LEAST, 39, MOST, 30, 7, 96, 2]
    seq = [0, 1, 2, 4, 2, 3, 4, LEAST, 5]
    codes, scales, table = pool.gpu()
    q_out = torch.full_like(q, 7.0)
    E.op_kv8_write(codes, scales, table, k, k, _ints(start), _ints(pos0), max_len, q=q, q_out=q_out, sections=(20, 12),
                   axis_pos=torch.from_numpy(axis).cuda(), cos=torch.from_numpy(cos).cuda(),
                   sin=torch.from_numpy(sin).cuda(), seq=_ints(seq))
    wc, ws = pool.codes.copy(), pool.scales.copy()
    wq = R.write(wc, ws, pool.table, k64, k64, start, pos0, max_len, [20, 12], axis, cos, sin, seq, q64)
    _same_codes(_bits(codes), wc)
    np.testing.assert_array_equal(scales.cpu().numpy(), ws)
    assert np.array_equal(q_out.double().cpu().numpy().reshape(wq.shape) == 7.0, np.isnan(wq))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("max_q,max_kv", [(1, 100), (3, 64), (40, 100), (40, 1 << 30)])
def test_attn_of_any_numbers(dtype, max_q, max_kv):
    rng = np.random.default_rng(72)
    lens = [40, 70, 100, 33]
    pool = Pool(73, lens, 2, 64)
    pool.table[2] = ([LEAST, MOST, pool.table[2, 2], -1, pool.nb, pool.table[2, 5]] + [0] * pool.table.shape[1])[
        :pool.table.shape[1]]
    rows = 60
    start = [5, 9, LEAST, 3, 17, MOST, 20, -4, 40, 2 ** 30]
    kv_len = [40, 70, LEAST, MOST, -1, 33, 100, 40, 2]
    seq = [0, 1, 2, 3, 2, 3, 2, LEAST, MOST]
    q, q64 = _rows(rng, rows, 4, 64, DT[dtype])
    codes, scales, table = pool.gpu()
    out = torch.full_like(q, 7.0)
    # sequences that overlap in their rows write the same rows: those are not looked at
    E.op_kv8_attn(codes, scales, table, q, out, _ints(start), _ints(kv_len), max_q, max_kv, seq=_ints(seq))
    got = out.double().cpu().numpy().reshape(q64.shape)
    count = np.zeros(rows, int)
    for i in range(9):
        r0 = min(max(start[i], 0), rows)
        count[r0:r0 + max(0, min(min(max(start[i + 1], 0), rows) - r0, max_q))] += 1
    want, bound = R.attend(pool.codes, pool.scales, pool.table, q64, start, kv_len, max_q, max_kv, True, 0.125, seq,
                           dtype == "bf16")
    # a page of no tokens holds NaN: rows that see one are NaN
    bound[count > 1] = np.inf
    bad = np.isnan(want) & ~np.isnan(bound) | np.isnan(bound) & (count[:, None, None] > 0)
    assert np.all(got[count == 0] == 7.0)
    ok = ~bad & (count == 1)[:, None, None] & ~np.isnan(want)
    assert np.all(np.abs(got - want)[ok] <= bound[ok])
    assert ok.any()


@gpu
@pytest.mark.parametrize("ql", [1, 40])
def test_pool_past_four_gib(ql):
    """Pages whose codes lie past 2^32 bytes, and past 2^31, beside the same sequence in low pages."""
    hkv, hd, n = 8, 128, 75
    nb = (1 << 32) // (2 * hkv * 16 * hd) + 64
    codes = torch.zeros((nb, 2, hkv, 16 * hd), dtype=torch.uint8, device="cuda")
    scales = torch.ones((nb, 2, hkv), device="cuda")
    pages = (n + 15) // 16
    table = torch.tensor([list(range(pages)), list(range(nb - pages, nb)), list(range(nb // 2 + 7, nb // 2 + 7 + pages))],
                         dtype=torch.int32, device="cuda")
    k, v = (torch.randn((n, hkv * hd), device="cuda").bfloat16().repeat(3, 1) for _ in range(2))
    for lo, hi in ((0, 60), (60, 61), (61, n)):            # prompts and a token
        m = hi - lo
        rows = torch.cat([torch.arange(lo, hi) + i * n for i in range(3)])
        E.op_kv8_write(codes, scales, table, k[rows], v[rows], _ints([0, m, 2 * m, 3 * m]), _ints([lo] * 3), m)
    t = table.long()
    assert codes[t[0]].any()
    assert torch.equal(codes[t[0]], codes[t[1]]) and torch.equal(codes[t[0]], codes[t[2]])
    assert torch.equal(scales[t[0]], scales[t[1]])
    assert not codes[pages:nb // 2].any()
    q = torch.randn((ql, 2 * hkv * hd), device="cuda").bfloat16().repeat(3, 1)
    out = torch.empty_like(q)
    E.op_kv8_attn(codes, scales, table, q, out, _ints([0, ql, 2 * ql, 3 * ql]), _ints([n] * 3), ql, n)
    assert torch.equal(out[:ql], out[ql:2 * ql]) and torch.equal(out[:ql], out[2 * ql:])
    assert out.abs().sum() > 0


@gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_write_token_by_token_grows_the_scale(hd):
    """Forty tokens one at a time, sizes over 2^-30 .. 2^30: every step's bytes, and, where the sizes do not
    underflow, the bytes that one call for all gives."""
    rng = np.random.default_rng(12)
    pool = Pool(13, [0], 2, hd, room=48)
    codes, scales, table = pool.gpu()
    wc, ws = pool.codes.copy(), pool.scales.copy()
    size = np.exp2(rng.uniform(-30, 30, 40)) * (np.arange(40) % 7 != 3)
    x = torch.from_numpy((rng.standard_normal((2, 40, 2 * hd)) * size[:, None])).float().cuda()
    for j in range(40):
        k, v = x[0, j:j + 1], x[1, j:j + 1]
        E.op_kv8_write(codes, scales, table, k, v, _ints([0, 1]), _ints([j]), 1)
        R.write(wc, ws, pool.table, k.double().cpu().numpy().reshape(1, 2, hd),
                v.double().cpu().numpy().reshape(1, 2, hd), [0, 1], [j], 1)
        _same_codes(_bits(codes), wc)
        np.testing.assert_array_equal(scales.cpu().numpy(), ws)


@gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_write_in_parts_is_the_write_at_once(hd):
    """Values within 2^12 of each other lose nothing when a page's scale grows: any split gives the same values."""
    rng = np.random.default_rng(14)
    n = 61
    x = torch.from_numpy(rng.uniform(0.5, 1.0, (2, n, 3 * hd)) * rng.choice([-1, 1], (2, n, 3 * hd)) *
                         np.exp2(rng.integers(0, 6, (2, n, 1)))).bfloat16().cuda()
    whole = Pool(15, [0], 3, hd, room=n).gpu()
    E.op_kv8_write(*whole, x[0], x[1], _ints([0, n]), _ints([0]), n)
    for cuts in ([0, 1, n], [0, 7, 8, 30, n], list(range(n + 1))):
        part = Pool(15, [0], 3, hd, room=n).gpu()
        for a, b in zip(cuts, cuts[1:]):
            E.op_kv8_write(*part, x[0, a:b], x[1, a:b], _ints([0, b - a]), _ints([a]), b - a)
        vw = R.CODE[_bits(whole[0])] * whole[1].cpu().numpy()[..., None]
        vp = R.CODE[_bits(part[0])] * part[1].cpu().numpy()[..., None]
        np.testing.assert_array_equal(vw, vp)


@gpu
def test_write_special_values():
    """NaN, infinities and 2^127 become NaN and leave the scale to the others; zeros, the largest and the least."""
    hd = 64
    pool = Pool(16, [0], 1, hd, room=64)
    x = np.ones((4, hd), np.float32)
    x[0, 3], x[0, 5], x[0, 9] = np.nan, np.inf, -np.inf
    x[1, :] = 0
    x[2, :] = 1e-38
    x[3, 7], x[3, 8] = 2.0 ** 127, -(2.0 ** 126)
    for lo, hi in ((0, 1), (1, 2), (2, 3), (3, 4), (0, 4)):
        codes, scales, table = pool.gpu()
        wc, ws = pool.codes.copy(), pool.scales.copy()
        t = torch.from_numpy(x[lo:hi]).cuda()
        E.op_kv8_write(codes, scales, table, t, t, _ints([0, hi - lo]), _ints([0]), hi - lo)
        x64 = x[lo:hi].astype(np.float64).reshape(hi - lo, 1, hd)
        R.write(wc, ws, pool.table, x64, x64, [0, hi - lo], [0], hi - lo)
        _same_codes(_bits(codes), wc)
        np.testing.assert_array_equal(scales.cpu().numpy(), ws)


@gpu
def test_write_rotates_in_place():
    rng = np.random.default_rng(17)
    pool = Pool(18, [0], 2, 128, room=40)
    k, _ = _rows(rng, 33, 2, 128, torch.bfloat16)
    q, _ = _rows(rng, 33, 4, 128, torch.bfloat16)
    cos, sin = (torch.from_numpy(t).cuda() for t in _tables(64, 128))
    apart = torch.empty_like(q)
    for out in (apart, q):
        E.op_kv8_write(*pool.gpu(), k, k, _ints([0, 33]), _ints([0]), 33, q=q, q_out=out, sections=(64,), cos=cos, sin=sin)
    assert torch.equal(apart, q)


def _check_attn(pool, dt, hq, lens, ql, causal, seed, pad=0, seq=None, outside=2, max_kv=None, scale=None, q_scale=1.0,
                max_q=None, workspace=None, only=None):
    rng = np.random.default_rng(seed)
    hd = pool.hd
    rows = sum(ql) + outside
    start = np.concatenate([[0], np.cumsum(ql)])
    q, _ = _rows(rng, rows, hq, hd, dt, pad)
    q *= q_scale
    q64 = q.double().cpu().numpy().reshape(rows, hq, hd)
    codes, scales, table = pool.gpu()
    out = torch.full((rows, hq * hd + 2 * pad), 7.0, dtype=dt, device="cuda")[:, :hq * hd]
    mq = max(list(ql) + [1]) if max_q is None else max_q
    mk = max(list(lens) + [1]) if max_kv is None else max_kv
    E.op_kv8_attn(codes, scales, table, q, out, _ints(start), _ints(lens), mq, mk, causal=causal, scale=scale,
                  seq=None if seq is None else _ints(seq), workspace=workspace)
    want, bound = R.attend(pool.codes, pool.scales, pool.table, q64, list(start), list(lens), mq, mk, causal,
                           hd ** -0.5 if scale is None else scale, seq, dt == torch.bfloat16, only)
    got = out.double().cpu().numpy().reshape(want.shape)
    _held(got, want, bound)
    return out


def _held(got, want, bound):
    outside = np.isnan(bound) & ~np.isnan(got)
    assert np.all(got[outside] == 7.0)          # rows of no sequence (want NaN there too)
    inside = ~np.isnan(bound) & ~np.isinf(bound)
    bad = ~(np.abs(got - want) <= bound) & inside
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], bound[bad][:5])
    err = np.linalg.norm((got - want)[inside]) / max(np.linalg.norm(want[inside]), 1e-30)
    print(f"rel {err:.2e}, largest share of the bound {np.max(np.abs(got - want)[inside] / np.maximum(bound[inside], 1e-30)):.2f}")


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 4, 64), (6, 2, 128), (16, 1, 128), (15, 3, 64), (40, 2, 64)])
def test_attn_decode(dtype, hq, hkv, hd):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 100, 0, 128, 129, 257, 300]
    pool = Pool(20, lens, hkv, hd)
    _check_attn(pool, DT[dtype], hq, lens, [1] * len(lens), True, 21, pad=8)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 4, 64), (6, 2, 128), (8, 1, 64)])
def test_attn_prompt(dtype, causal, hq, hkv, hd):
    lens, ql = [1, 17, 70, 5, 40, 0, 33, 64], [1, 17, 50, 9, 0, 3, 2, 64]     # 9 rows on 5 keys: four see none
    pool = Pool(22, lens, hkv, hd)
    _check_attn(pool, DT[dtype], hq, lens, ql, causal, 23, pad=8)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ql", [1, 3, 8, 20, 70])
def test_attn_long_keys_are_cut_and_joined(dtype, ql):
    lens = [2100, 900, 1]
    pool = Pool(24, lens, 2, 128)
    _check_attn(pool, DT[dtype], 4, lens, [ql, ql, 1], True, 25)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
def test_attn_decode_many_pairs(dtype, hd):
    """Enough (sequence, KV head) pairs for a wave each; 1030 of them end inside a workgroup."""
    lens = [(i * 7) % 61 for i in range(103)]
    pool = Pool(60, lens, 10, hd)
    _check_attn(pool, DT[dtype], 20, lens, [1] * 103, True, 61, only=set(range(0, 103, 5)) | {101, 102})


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,causal", [(64, True), (128, True), (128, False)])
def test_attn_prompt_many_rows(dtype, hd, causal):
    """Rows and keys enough for the tallest tiles, keys past what LDS lists at a time, ragged; a sample of the rows."""
    lens, ql = [5000, 4111, 300], [4500, 4097, 290]
    pool = Pool(62, lens, 8, hd)
    rng = np.random.default_rng(63)
    rows = sum(ql)
    only = {0, 1, 4499, 4500, 8596, 8597, rows - 1} | set(rng.integers(0, rows, 12).tolist())
    _check_attn(pool, DT[dtype], 8, lens, ql, causal, 64, only=only)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attn_prompt_middle(dtype):
    """Workgroups of 64 rows."""
    lens, ql = [150, 90, 33, 170], [150, 70, 33, 100]
    pool = Pool(65, lens, 44, 64)
    _check_attn(pool, DT[dtype], 44, lens, ql, True, 66, only=set(range(0, sum(ql), 29)))


@gpu
def test_attn_one_long_sequence():
    lens = [20011]
    pool = Pool(26, lens, 1, 64)
    _check_attn(pool, torch.bfloat16, 2, lens, [1], True, 27)
    _check_attn(pool, torch.float32, 2, lens, [2], True, 28)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attn_strong_scores(dtype):
    """Weights on few keys, and sizes that differ by page."""
    lens = [200, 77]
    pool = Pool(29, lens, 2, 64, spread=6.0)
    _check_attn(pool, DT[dtype], 4, lens, [1, 1], True, 30, q_scale=4.0)
    _check_attn(pool, DT[dtype], 4, lens, [60, 30], True, 31, q_scale=4.0, scale=0.5)
    _check_attn(pool, DT[dtype], 4, lens, [60, 30], False, 32, scale=1e-6)
    pool = Pool(69, lens, 2, 128, spread=6.0)
    _check_attn(pool, DT[dtype], 4, lens, [60, 30], True, 31, q_scale=4.0, scale=0.5)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ql", [1, 40])
@pytest.mark.parametrize("hd", [64, 128])
def test_attn_rows_of_all_sizes(dtype, ql, hd):
    """Queries whose elements, and whose rows, are powers of two apart; rows of zeros and of the least values."""
    pool = Pool(67, [90, 41], 2, hd)
    rng = np.random.default_rng(68)
    size = np.exp2(rng.integers(-20, 1, (2 * ql, 4 * hd)) + rng.integers(-8, 4, (2 * ql, 1)))
    size[::7] = 0.0
    size[3::7] = 1e-37
    q = torch.from_numpy(rng.standard_normal((2 * ql, 4 * hd)) * size).to(DT[dtype]).cuda()
    codes, scales, table = pool.gpu()
    out = torch.empty_like(q)
    E.op_kv8_attn(codes, scales, table, q, out, _ints([0, ql, 2 * ql]), _ints([90, 41]), ql, 90)
    q64 = q.double().cpu().numpy().reshape(2 * ql, 4, hd)
    want, bound = R.attend(pool.codes, pool.scales, pool.table, q64, [0, ql, 2 * ql], [90, 41], ql, 90, True, hd ** -0.5,
                           bf16=dtype == "bf16")
    _held(out.double().cpu().numpy().reshape(want.shape), want, bound)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ql", [1, 40])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("up", [-92, -60, 60, 112])
def test_attn_sizes_of_keys_and_queries_that_cancel(dtype, ql, hd, up):
    """Keys 2^up times as large and queries 2^-up: the scores are ordinary."""
    lens = [90, 41]
    pool = Pool(83, lens, 2, hd)
    pool.scales[:, 0] *= 2.0 ** up
    _check_attn(pool, DT[dtype], 4, lens, [ql, ql], True, 84, q_scale=2.0 ** -up)


@gpu
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("up", [-92, 0, 112])
def test_attn_sizes_that_cancel_in_tall_tiles(hd, up):
    """The same with 32 rows a wave: 260 sequences of 20 rows, all on one sequence's keys."""
    pool = Pool(87, [90], 2, hd)
    pool.scales[:, 0] *= 2.0 ** up
    n = 260
    _check_attn(pool, torch.bfloat16, 4, [90] * n, [20] * n, True, 88, q_scale=2.0 ** -up, seq=[0] * n, max_kv=1024,
                only=set(range(40)) | set(range(20 * n - 20, 20 * n)))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ql", [1, 40])
@pytest.mark.parametrize("up", [-90, 100])
def test_attn_values_near_the_ends_of_the_range(dtype, ql, up):
    """Values 2^up times as large: weights of up to 2^10 over 90 keys leave the sums of 2^100 ones below 2^128."""
    lens = [90, 41]
    pool = Pool(85, lens, 2, 128)
    pool.scales[:, 1] *= 2.0 ** up
    _check_attn(pool, DT[dtype], 4, lens, [ql, ql], True, 86, scale=1.0)


@gpu
@pytest.mark.parametrize("causal", [True, False])
def test_attn_bound_far_above_the_rows(causal):
    """A bound of 6 M query rows for sequences of 20 and 40: 786432 workgroups, most with nothing to do."""
    lens = [60, 90]
    pool = Pool(81, lens, 4, 64)
    _check_attn(pool, torch.bfloat16, 4, lens, [20, 40], causal, 82, max_q=6 << 20)


@gpu
@pytest.mark.parametrize("ql", [1, 40])
def test_attn_keeps_to_its_bounds(ql):
    """Unknown table rows are empty, pages that are none are not seen, row
    ranges and lengths are cut."""
    lens = [60, 90, 33, 48]
    pool = Pool(33, lens, 2, 64)
    pool.table[1, 2], pool.table[1, 5] = pool.nb, -7
    pool.table[2, :] = -1
    n = [ql] * 4
    _check_attn(pool, torch.bfloat16, 4, lens, n, True, 34)
    _check_attn(pool, torch.bfloat16, 4, lens, n, False, 35, seq=[3, 4, -1, 0])
    _check_attn(pool, torch.bfloat16, 4, lens, n, True, 36, max_kv=50, outside=-ql)
    _check_attn(pool, torch.bfloat16, 4, [60, 90, 10 ** 9, -3], n, True, 37, max_kv=200, max_q=max(1, ql - 3))


@gpu
@pytest.mark.parametrize("copies", [1, 300])
@pytest.mark.parametrize("ql", [1, 5, 40])
@pytest.mark.parametrize("hkv,hd", [(2, 64), (4, 64), (2, 128)])
def test_attn_nan_counts_only_where_it_is_seen(ql, hkv, hd, copies):
    """NaN keys and values: rows that see them are NaN (a value's in its dim
    alone), rows that do not are what they are without.  Copies of the second
    sequence bring the kernels of large batches."""
    n = 70
    rng = np.random.default_rng(38)
    pool = Pool(39, [n, n], hkv, hd)
    clean = pool.codes.copy()

    def put(t, dim, value):
        pg = pool.table[0, t // 16]
        pool.codes[pg, value, 0, R.order(hd, value)[t % 16, dim]] = 0xFF
    put(n - 2, 5, 1)          # seen by the last two rows only
    put(n - 20, 17, 1)
    put(n - 1, 3, 0)          # the last row is NaN as a whole
    seq = [0] + [1] * copies
    start = [ql * i for i in range(copies + 2)]
    q, q64 = _rows(rng, start[-1], 4, hd, torch.bfloat16)
    res = []
    for c in (clean, pool.codes):
        out = torch.empty_like(q)
        E.op_kv8_attn(torch.from_numpy(c).cuda(), torch.from_numpy(pool.scales).cuda(), torch.from_numpy(pool.table).cuda(),
                      q, out, _ints(start), _ints([n] * len(seq)), ql, n, seq=_ints(seq))
        res.append(out.double().cpu().numpy().reshape(len(seq), ql, 4, hd))
    want = res[0].copy()
    mine = 4 // hkv
    for j in range(ql):
        sees = n - ql + j
        if sees >= n - 2:
            want[0, j, :mine, 5] = np.nan
        if sees >= n - 20:
            want[0, j, :mine, 17] = np.nan
        if sees >= n - 1:
            want[0, j, :mine] = np.nan
    assert np.array_equal(np.isnan(want), np.isnan(res[1]))
    np.testing.assert_array_equal(want, res[1])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ql,copies", [(1, 1), (6, 1), (40, 1), (40, 300), (1, 600)])
def test_attn_queries_that_are_not_finite(dtype, hd, ql, copies):
    """A NaN or an infinity in a query row makes that row and head NaN and leaves the others as they are."""
    pool = Pool(74, [70], 2, hd)
    n = copies + 1
    start = [ql * i for i in range(n + 1)]
    q = torch.randn((n * ql, 4 * hd), device="cuda").to(DT[dtype])
    codes, scales, table = pool.gpu()
    res = []
    for bad in (False, True):
        if bad:
            q[0, 3], q[ql - 1, hd + 7], q[-1, 2 * hd + 1] = float("nan"), float("inf"), float("-inf")
        out = torch.empty_like(q)
        E.op_kv8_attn(codes, scales, table, q, out, _ints(start), _ints([70] * n), ql, 70, seq=_ints([0] * n))
        res.append(out.reshape(n * ql, 4, hd))
    hit = torch.zeros((n * ql, 4), dtype=torch.bool, device="cuda")
    hit[0, 0] = hit[ql - 1, 1] = hit[-1, 2] = True
    assert torch.isnan(res[1][hit]).all()
    assert torch.equal(res[0][~hit], res[1][~hit])


@gpu
@pytest.mark.parametrize("ql", [1, 33])
def test_attn_workspace_serves_call_after_call(ql):
    """One workspace, calls of several shapes that it is large enough for, results the same each time."""
    lens = [3000, 1200]
    pool = Pool(40, lens, 2, 64)
    codes, scales, table = pool.gpu()
    q = torch.randn((2 * ql, 256), device="cuda").bfloat16()
    ws = E.kv8_attn_workspace(codes, table, q, 2, ql, 3000)
    assert ws.numel() > 0
    first = None
    for _ in range(3):
        out = torch.empty_like(q)
        E.op_kv8_attn(codes, scales, table, q, out, _ints([0, ql, 2 * ql]), _ints(lens), ql, 3000, workspace=ws)
        first = out if first is None else first
        assert torch.equal(first, out)
    fresh = torch.empty_like(q)
    E.op_kv8_attn(codes, scales, table, q, fresh, _ints([0, ql, 2 * ql]), _ints(lens), ql, 3000)
    assert torch.equal(first, fresh)
    with pytest.raises(E.EbrlError):
        E.op_kv8_attn(codes, scales, table, q, fresh, _ints([0, ql, 2 * ql]), _ints(lens), ql, 3000, workspace=ws[:-16])


@gpu
def test_decode_loop_in_a_graph():
    """Write and attention of a token in a captured graph, replayed with new
    rows and lengths beside eager work, against eager calls on another cache;
    two graphs with a workspace each."""
    lens, steps, hq, hkv, hd = [50, 700, 15], 5, 4, 2, 128
    pool = Pool(41, lens, hkv, hd, room=steps)
    cos, sin = (torch.from_numpy(t).cuda() for t in _tables(800, hd))
    start = _ints([0, 1, 2, 3])
    mx = max(lens) + steps
    x = torch.randn((steps, 3, (hq + 2 * hkv) * hd), device="cuda").bfloat16()

    def step(cache, qkv, q, out, pos, kvl, ws):
        E.op_kv8_write(*cache, qkv[:, hq * hd:(hq + hkv) * hd], qkv[:, (hq + hkv) * hd:], start, pos, 1,
                       q=qkv[:, :hq * hd], q_out=q, sections=(hd // 2,), cos=cos, sin=sin)
        E.op_kv8_attn(*cache, q, out, start, kvl, 1, mx, workspace=ws)

    eager, want = pool.gpu(), []
    for j in range(steps):
        q, out = torch.empty((3, hq * hd), device="cuda").bfloat16(), torch.empty((3, hq * hd), device="cuda").bfloat16()
        step(eager, x[j], q, out, _ints(lens) + j, _ints(lens) + j + 1, None)
        want.append(out)
    graphs = []
    for _ in range(2):
        s = {"cache": pool.gpu(), "qkv": x[0].clone(), "q": torch.empty_like(want[0]), "out": torch.empty_like(want[0]),
             "pos": _ints(lens), "kvl": _ints(lens) + 1}
        s["ws"] = E.kv8_attn_workspace(s["cache"][0], s["cache"][2], s["q"], 3, 1, mx)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            step(s["cache"], s["qkv"], s["q"], s["out"], s["pos"], s["kvl"], s["ws"])
        graphs.append((g, s))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for j in range(steps):
        for (g, s), st in zip(graphs, streams):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                s["qkv"].copy_(x[j])
                s["pos"].copy_(_ints(lens) + j)
                s["kvl"].copy_(_ints(lens) + j + 1)
                g.replay()
        torch.cuda.synchronize()
        for _, s in graphs:
            assert torch.equal(s["out"], want[j]), j
    for _, s in graphs:
        assert np.array_equal(_bits(s["cache"][0]), _bits(eager[0]))
        np.testing.assert_array_equal(s["cache"][1].cpu().numpy(), eager[1].cpu().numpy())


@gpu
def test_prompt_then_tokens_match_the_definition():
    """A prompt's rows written and attended to in two parts, then tokens, every output against the float64 form."""
    hq, hkv, hd, n = 4, 2, 64, 90
    rng = np.random.default_rng(42)
    pool = Pool(43, [0, 0], hkv, hd, room=n)
    cos, sin = _tables(n, hd)
    dc, ds = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    codes, scales, table = pool.gpu()
    wc, ws = pool.codes.copy(), pool.scales.copy()
    for a, b in ((0, 37), (37, 80), (80, 81), (81, 82), (82, 90)):
        m = b - a
        q, q64 = _rows(rng, 2 * m, hq, hd, torch.bfloat16)
        k, k64 = _rows(rng, 2 * m, hkv, hd, torch.bfloat16)
        v, v64 = _rows(rng, 2 * m, hkv, hd, torch.bfloat16)
        axis = rng.integers(0, n, (2 * m, 3)).astype(np.int32)
        start = [0, m, 2 * m]
        out = torch.empty_like(q)
        E.op_kv8_write(codes, scales, table, k, v, _ints(start), _ints([a, a]), m, q=q, q_out=q, sections=(12, 10, 10),
                       axis_pos=torch.from_numpy(axis).cuda(), cos=dc, sin=ds)
        E.op_kv8_attn(codes, scales, table, q, out, _ints(start), _ints([b, b]), m, n)
        R.write(wc, ws, pool.table, k64, v64, start, [a, a], m, [12, 10, 10], axis, cos, sin)
        _same_codes(_bits(codes), wc)
        qr = q.double().cpu().numpy().reshape(2 * m, hq, hd)
        want, bound = R.attend(wc, ws, pool.table, qr, start, [b, b], m, n, True, hd ** -0.5)
        _held(out.double().cpu().numpy().reshape(want.shape), want, bound)


@gpu
def test_calls_on_another_stream():
    pool = Pool(44, [300, 40], 2, 64)
    codes, scales, table = pool.gpu()
    q = torch.randn((2, 256), device="cuda").bfloat16()
    st, kl = _ints([0, 1, 2]), _ints([300, 40])
    want = torch.empty_like(q)
    E.op_kv8_attn(codes, scales, table, q, want, st, kl, 1, 300)
    s = torch.cuda.Stream()
    got = torch.empty_like(q)
    ws = E.kv8_attn_workspace(codes, table, q, 2, 1, 300)
    torch.cuda.synchronize()
    E.op_kv8_attn(codes, scales, table, q, got, st, kl, 1, 300, workspace=ws, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(want, got)
    with torch.cuda.stream(s):
        E.op_kv8_attn(codes, scales, table, q, got.zero_(), st, kl, 1, 300)
    s.synchronize()
    assert torch.equal(want, got)


# (sequences, query rows of each, keys, keys of a step's size, bound on the keys): the four ways to cut a call, with
# 16 rows a wave (of which head dim 128 gives K's codes to the scaled product) and 32, in one part and in several
LADDERS = {"decode": (1, 1, 60, 1, 60), "decode-wave": (600, 1, 60, 1, 60), "decode-parts": (1, 3, 2100, 40, 2100),
           "prompt": (1, 40, 60, 1, 60), "prompt-parts": (1, 24, 2100, 40, 2100), "prompt-64": (260, 33, 60, 1, 60),
           "prompt-128": (260, 20, 60, 1, 1024)}


def _ladder(kind, hd, sign, up, dt, causal=True):
    """Keys in steps, each step's scores above those of the step before by a sixtieth of the largest, queries of one size
    in all dims: a row's result is the value of the last step that it sees.  Scores in log2 go up to about 2^up (sign 1)
    or start there (sign -1).  Returns (got, want), [rows, heads, hd]."""
    n, ql, keys, tie, bound = LADDERS[kind]
    rng = np.random.default_rng(100 + up)
    hkv, grp = 2, 2
    pool = Pool(101, [0], hkv, hd, room=keys)
    step = np.arange(keys) // tie
    count = step + 1 if sign > 0 else step[-1] + 1 - step
    assert count.max() <= hd
    k = sign * (np.arange(hd) < count[:, None])[:, None, :] * np.ones((1, hkv, 1)) * 2.0 ** (up // 2)
    v = rng.standard_normal((step[-1] + 1, hkv, hd))[step]
    R.write(pool.codes, pool.scales, pool.table, k, v, [0, keys], [0], keys)
    size = rng.uniform(1, 2, (n * ql, hkv * grp, 1)) * 2.0 ** (up - up // 2) / (60 * hd ** -0.5)
    q = torch.from_numpy((size * np.ones(hd)).reshape(n * ql, -1)).to(dt).cuda()
    codes, scales, table = pool.gpu()
    out = torch.full_like(q, 7.0)
    E.op_kv8_attn(codes, scales, table, q, out, _ints(ql * np.arange(n + 1)), _ints([keys] * n), ql, bound, causal=causal,
                  seq=_ints([0] * n))
    _, V, _ = R.gather(pool.codes, pool.scales, pool.table[0], keys)
    last = keys - ql + np.arange(ql) if causal else np.full(ql, keys - 1)
    want = np.tile(np.repeat(V[last], grp, axis=1), (n, 1, 1))
    return out.double().cpu().numpy().reshape(want.shape), want


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kind", list(LADDERS))
def test_attn_large_scores_give_the_largest_keys_value(kind, hd, dtype):
    """Scores of 2^20 to 2^100 in log2, of either sign.  A sixtieth of 2^20 is more than any weight's range: one step's
    value is all of the result, off by the rounding of the weights (one bf16 term: the sum takes them as rounded; two: 2^-17
    of them; three: 2^-24), of up to 40 sums of them and of the result."""
    for up in (20, 24, 25, 27, 30, 33, 40, 60, 100):
        for sign in (1, -1):
            for causal in (True, False):
                got, want = _ladder(kind, hd, sign, up, DT[dtype], causal)
                tol = 2.0 ** -8 + 2.0 ** -16 + 2.0 ** -17 if dtype == "bf16" else 2.0 ** -16
                bad = ~(np.abs(got - want) <= tol * np.abs(want))
                assert not bad.any(), (up, sign, causal, got[bad][:4], want[bad][:4])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kind", list(LADDERS))
def test_attn_scores_that_are_all_minus_infinity(kind, hd, dtype):
    """A row that sees keys, every score of which is -infinity, is NaN: it is no row that sees none.  One score that is
    not leaves it that key's value.  Rows that see no key stay zeros; the others hold to the rounding of two weights."""
    n, ql, keys, _, bound = LADDERS[kind]
    rng = np.random.default_rng(110)
    pool = Pool(111, [0], 2, hd, room=keys)
    k = rng.uniform(1, 2, (keys, 2, hd)) * 2.0 ** 70
    k[0, :, 7] = 0
    R.write(pool.codes, pool.scales, pool.table, k, rng.standard_normal((keys, 2, hd)), [0, keys], [0], keys)
    codes, scales, table = pool.gpu()
    _, V, _ = R.gather(pool.codes, pool.scales, pool.table[0], keys)
    q = torch.from_numpy(rng.uniform(1, 2, ((n + 1) * ql, 4 * hd)) * 2.0 ** -76).to(DT[dtype]).cuda()
    end = n * ql                                  # a last sequence, whose first rows see no key
    lens = [keys] * n + [max(0, ql - 3)]
    res = []
    for bad in (False, True):
        if bad:
            q[0, 3] = q[end, 3] = float("-inf")   # head 0
            q[ql // 2, hd:2 * hd] = -2.0 ** 70    # head 1: finite, every score past the range
            q[ql - 1, 2 * hd:3 * hd] = 0          # head 2: all but key 0's
            q[ql - 1, 2 * hd + 7] = -2.0 ** 70
        out = torch.full_like(q, 7.0)
        E.op_kv8_attn(codes, scales, table, q, out, _ints(ql * np.arange(n + 2)), _ints(lens), ql, bound,
                      seq=_ints([0] * (n + 1)))
        res.append(out.double().cpu().numpy().reshape(-1, 4, hd))
    want = res[0]
    assert np.all(want[end:end + min(ql, 3)] == 0)
    want[0, 0] = want[ql // 2, 1] = np.nan
    want[ql - 1, 2] = V[0, 1]
    assert np.array_equal(np.isnan(res[1]), np.isnan(want))
    assert np.nanmax(np.abs(res[1] - want)) <= 2.0 ** -6 * np.abs(V).max()


@pytest.mark.parametrize("dtype", [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.bool])
def test_binding_refuses_codes_of_other_formats(dtype):
    """Bytes are taken as e4m3 codes; a type that says they are something else is refused."""
    codes, scales = E.kv8_alloc(4, 2, 64, device="cpu")
    other = codes.view(torch.uint8).view(dtype)
    table = torch.zeros((1, 4), dtype=torch.int32)
    k = torch.zeros((1, 128), dtype=torch.bfloat16)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    with pytest.raises(E.EbrlError, match="codes are"):
        E.op_kv8_write(other, scales, table, k, k, i32(0, 1), i32(0), 1)
    with pytest.raises(E.EbrlError, match="codes are"):
        E.op_kv8_attn(other, scales, table, k, k.clone(), i32(0, 1), i32(1), 1, 1)
    with pytest.raises(E.EbrlError, match="codes are"):
        E.kv8_attn_workspace(other, table, k, 1, 1, 1)
    for raw in (torch.uint8, torch.int8, torch.float8_e4m3fn):
        with pytest.raises(E.EbrlError, match="not on a GPU"):
            E.op_kv8_write(codes.view(torch.uint8).view(raw), scales, table, k, k, i32(0, 1), i32(0), 1)
        assert E.kv8_attn_workspace(codes.view(torch.uint8).view(raw), table, k, 1, 1, 1).numel() == 0


def test_binding_takes_one_row_of_any_stride():
    """A single row's stride says nothing: it is not held to the 16 bytes that rows are apart by."""
    buf = torch.zeros((3, 130), dtype=torch.bfloat16)
    assert E._kv8_rows("k", buf[:1, :128], torch.bfloat16, -1, 1, 128) == (buf.data_ptr(), 128)
    assert E._kv8_rows("k", buf[:, :128], torch.bfloat16, -1, 3, 128) == (buf.data_ptr(), 130)
    codes, scales = E.kv8_alloc(4, 2, 64, device="cpu")
    k = buf[:1, :128]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    with pytest.raises(E.EbrlError, match="not on a GPU"):
        E.op_kv8_write(codes, scales, torch.zeros((1, 4), dtype=torch.int32), k, k, i32(0, 1), i32(0), 1)


def test_counts_that_pass_64_bits_are_refused():
    """Sequences, heads and rows whose number of workgroups wraps round to a few, or to none."""
    big = dict(ldq=1 << 39, ldo=1 << 39)
    for heads, n, q in ((1 << 24, 1 << 30, 1 << 16), (1 << 20, (1 << 31) - 1, 1 << 29), (1 << 30, 1 << 30, 128),
                        (1 << 20, 1 << 22, 1 << 29)):
        c = _cache(kv_heads=heads)
        a = _attn_args(n=n, rows=5, max_q_len=q, q_heads=heads, **big)
        assert _attn(c, a) == -1, (heads, n, q)
        assert E.lib().ebrl_op_kv8_attn_workspace(ctypes.byref(c), ctypes.byref(a)) == -1, (heads, n, q)
    wide = dict(ldq=1 << 39, ldk=1 << 39, ldv=1 << 39, ldq_out=1 << 39)
    top = (1 << 31) - 1
    for heads, q_heads, n, rows in ((1 << 30, 0, 1 << 30, 1 << 30), (1 << 30, 1 << 30, 1, 16), (2, top, 1, 16),
                                    (1 << 20, 1 << 20, top, top)):
        a = _write_args(n=n, rows=rows, max_len=rows, q_heads=q_heads, **wide)
        assert E.lib().ebrl_op_kv8_write(ctypes.byref(_cache(kv_heads=heads)), ctypes.byref(a), None) == -1, (heads, n)


def _terms(p, n):
    """Weights as n bf16 terms, added up."""
    got = np.zeros_like(p)
    for _ in range(n):
        got += torch.from_numpy(p - got).bfloat16().double().numpy()
    return got


def _decode_case(seed, lens, hkv, hd, hq):
    pool = Pool(seed, lens, hkv, hd)
    q = torch.from_numpy(np.random.default_rng(seed + 1).standard_normal((len(lens), hq * hd))).bfloat16()
    return pool, q


def test_two_term_bound_tells_one_term_from_two():
    """A decode step whose weights were rounded to one bf16 term would leave the bound that two terms are held to."""
    lens, hkv, hd, hq = [300, 1000], 2, 64, 4
    pool, q = _decode_case(120, lens, hkv, hd, hq)
    q64 = q.double().numpy().reshape(len(lens), hq, hd)
    want, bound = R.attend(pool.codes, pool.scales, pool.table, q64, [0, 1, 2], lens, 1, 1000, True, hd ** -0.5,
                           weight_terms=2)
    for terms, holds in ((1, False), (2, True)):
        got = np.empty_like(want)
        for i, n in enumerate(lens):
            K, V, _ = R.gather(pool.codes, pool.scales, pool.table[i], n)
            for h in range(hq):
                s = K[:, h // 2] @ q64[i, h] * hd ** -0.5
                p = np.exp(s - s.max())
                got[i, h] = _terms(p, terms) @ V[:, h // 2] / p.sum()
        got = torch.from_numpy(got).bfloat16().double().numpy()
        assert bool(np.all(np.abs(got - want) <= bound)) == holds, terms


@gpu
@pytest.mark.parametrize("hq,hkv,hd,lens", [(4, 2, 64, [300, 1000, 77]), (6, 2, 128, [300, 1000, 77]), (16, 1, 128, [129]),
                                            (2, 1, 64, [9001]), (8, 1, 128, [6000, 4000]),
                                            (20, 10, 64, [(i * 7) % 61 for i in range(103)]),
                                            (20, 10, 128, [(i * 7) % 61 for i in range(103)])])
def test_attn_decode_weights_in_two_terms(hq, hkv, hd, lens):
    pool, q = _decode_case(122, lens, hkv, hd, hq)
    codes, scales, table = pool.gpu()
    out = torch.full_like(q, 7.0).cuda()
    n = len(lens)
    E.op_kv8_attn(codes, scales, table, q.cuda(), out, _ints(range(n + 1)), _ints(lens), 1, max(lens))
    want, bound = R.attend(pool.codes, pool.scales, pool.table, q.double().numpy().reshape(n, hq, hd), list(range(n + 1)),
                           lens, 1, max(lens), True, hd ** -0.5, weight_terms=2)
    _held(out.double().cpu().numpy().reshape(want.shape), want, bound)


@gpu
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype,copies,ql,bound", [("bf16", 260, 100, 1024), ("bf16", 300, 100, 120), ("bf16", 1, 100, 120),
                                                   ("fp32", 300, 100, 120), ("fp32", 1, 100, 120), ("fp32", 1, 5, 120),
                                                   ("fp32", 600, 5, 120)])
def test_attn_nan_in_every_page_of_a_step(dtype, copies, ql, bound, hd):
    """NaN values in the first, third and fourth page of a step of 64 keys, behind causal masks, and a NaN key; tiles of 128
    rows (the first case) and fp32 rows among them."""
    n, hkv = 120, 2
    rng = np.random.default_rng(130)
    pool = Pool(131, [n, n], hkv, hd)
    clean = pool.codes.copy()
    nans = {(40, 1), (55, 5), (70, 9), (100, 17), (115, 33), (118, hd - 1)}      # (token, dim)
    for t, dim in nans:
        pool.codes[pool.table[0, t // 16], 1, 0, R.order(hd, 1)[t % 16, dim]] = 0x7F
    pool.codes[pool.table[0, (n - 1) // 16], 0, 0, R.order(hd, 0)[(n - 1) % 16, 2]] = 0xFF
    seq = [0] + [1] * copies
    q, _ = _rows(rng, ql * len(seq), 4, hd, DT[dtype])
    res = []
    for c in (clean, pool.codes):
        out = torch.empty_like(q)
        E.op_kv8_attn(torch.from_numpy(c).cuda(), torch.from_numpy(pool.scales).cuda(), torch.from_numpy(pool.table).cuda(),
                      q, out, _ints(ql * np.arange(len(seq) + 1)), _ints([n] * len(seq)), ql, bound, seq=_ints(seq))
        res.append(out.double().cpu().numpy().reshape(len(seq), ql, 4, hd))
    want = res[0].copy()
    for j in range(ql):
        for t, dim in nans:
            if n - ql + j >= t:
                want[0, j, :2, dim] = np.nan
    want[0, ql - 1, :2] = np.nan
    np.testing.assert_array_equal(want, res[1])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kind", list(LADDERS))
def test_attn_leaves_rows_of_no_sequence(kind, hd, dtype):
    """Rows before the first sequence, past the bound of each and behind the last keep every byte; all others are written."""
    n, ql, keys, _, bound = LADDERS[kind]
    pool = Pool(140, [keys], 2, hd)
    codes, scales, table = pool.gpu()
    gap = 3
    start = 2 + (ql + gap) * np.arange(n + 1)
    q, _ = _rows(np.random.default_rng(141), int(start[-1]) + 4, 4, hd, DT[dtype])
    out = torch.full((q.shape[0], 4 * hd + 8), 7.0, dtype=DT[dtype], device="cuda")
    E.op_kv8_attn(codes, scales, table, q, out[:, :4 * hd], _ints(start), _ints([keys] * n), ql, bound,
                  seq=_ints([0] * n))
    mine = torch.zeros(q.shape[0], dtype=torch.bool)
    for r in start[:-1]:
        mine[r:r + ql] = True
    assert (out[~mine] == 7.0).all() and (out[:, 4 * hd:] == 7.0).all()
    assert torch.isfinite(out[mine]).all() and not (out[mine][:, :4 * hd] == 7.0).any()


def test_binding_refuses_shapes_past_32_bits():
    """Refused as other calls are, by the library's error."""
    codes = torch.empty((4, 2, 2, 1024), dtype=torch.uint8, device="meta")
    scales = torch.empty((4, 2, 2), device="meta")
    wide = torch.empty((1, 1 << 31), dtype=torch.int32, device="meta")
    tall = torch.empty((1 << 31, 2, 2, 1024), dtype=torch.uint8, device="meta")
    table = torch.empty((1, 4), dtype=torch.int32, device="meta")
    k = torch.empty((1, 128), dtype=torch.bfloat16, device="meta")
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device="meta")  # noqa: E731
    for c, s, t in ((codes, scales, wide), (tall, torch.empty((1 << 31, 2, 2), device="meta"), table)):
        with pytest.raises(E.EbrlError, match="32 bits"):
            E.op_kv8_write(c, s, t, k, k, i32(2), i32(1), 1)
        with pytest.raises(E.EbrlError, match="32 bits"):
            E.op_kv8_attn(c, s, t, k, torch.empty_like(k), i32(2), i32(1), 1, 1)
        with pytest.raises(E.EbrlError, match="32 bits"):
            E.kv8_attn_workspace(c, t, k, 1, 1, 1)
    rows = torch.empty((1 << 31, 128), dtype=torch.bfloat16, device="meta")
    with pytest.raises(E.EbrlError):
        E.kv8_attn_workspace(codes, table, rows, 1, 1, 1)


def test_workspace_refuses_queries_that_are_no_heads():
    codes, _ = E.kv8_alloc(4, 2, 64, device="cpu")
    table = torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(E.EbrlError, match="heads of 64"):
        E.kv8_attn_workspace(codes, table, torch.zeros((1, 190), dtype=torch.bfloat16), 1, 1, 1)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ql", [1, 40])
@pytest.mark.parametrize("hd", [64, 128])
def test_attn_pages_that_are_none_before_the_first(ql, hd, dtype):
    """Sequences of 200 pages of which the 1st, the 64th, the 65th, the 130th or none is there, in parts: a query of
    -infinity is NaN where a page is, zeros where none is; ordinary ones are a mean of that page's values."""
    n_pages, there = 200, [0, 63, 64, 129, None]
    rng = np.random.default_rng(150)
    pool = Pool(151, [16], 2, hd)
    page = pool.table[0, 0]
    table = np.full((5, n_pages), -1, np.int32)
    for i, p in enumerate(there):
        if p is not None:
            table[i, p] = page
    pool.table = table
    k = rng.uniform(1, 2, (16, 2, hd))
    v = rng.standard_normal((16, 2, hd))
    R.write(pool.codes, pool.scales, np.array([[page]]), k, v, [0, 16], [0], 16)
    codes, scales, dev = pool.gpu()
    q, q64 = _rows(rng, 5 * ql, 4, hd, DT[dtype])
    kv = [n_pages * 16] * 5
    start = [ql * i for i in range(6)]
    want, bound = R.attend(pool.codes, pool.scales, table, q64, start, kv, ql, max(kv), True, hd ** -0.5,
                           bf16=dtype == "bf16")
    out = torch.full_like(q, 7.0)
    E.op_kv8_attn(codes, scales, dev, q, out, _ints(start), _ints(kv), ql, max(kv))
    _held(out.double().cpu().numpy().reshape(want.shape), want, bound)
    assert (out[4 * ql:] == 0).all()
    q[:, 3] = float("-inf")
    E.op_kv8_attn(codes, scales, dev, q, out, _ints(start), _ints(kv), ql, max(kv))
    assert torch.isnan(out[:4 * ql, :hd]).all()
    assert (out[4 * ql:] == 0).all() and torch.isfinite(out[:, hd:]).all()


@gpu
@pytest.mark.parametrize("ql", [1, 40])
def test_attn_fp32_queries_at_the_end_of_bf16s_range(ql):
    """Queries enter as bf16 terms: one past bf16's largest number makes its row and head NaN, one just below does not."""
    pool = Pool(160, [70], 2, 64)
    pool.scales[:, 0] *= 2.0 ** -92
    codes, scales, table = pool.gpu()
    q = torch.randn((ql, 256), device="cuda")
    q[0, 3], q[ql - 1, 64 + 7] = 3.4e38, 3.38e38
    out = torch.empty_like(q)
    E.op_kv8_attn(codes, scales, table, q, out, _ints([0, ql]), _ints([70]), ql, 70)
    nan = torch.isnan(out).reshape(ql, 4, 64)
    assert nan[0, 0].all() and nan.sum() == 64


@gpu
@pytest.mark.parametrize("new", [[1, 1], [20, 3]])
def test_write_turns_keys_without_queries(new):
    past = [5, 30]
    pool = Pool(161, past, 2, 128, room=21)
    rng = np.random.default_rng(162)
    rows = sum(new)
    k, k64 = _rows(rng, rows, 2, 128, torch.bfloat16)
    cos, sin = _tables(64, 128)
    codes, scales, table = pool.gpu()
    E.op_kv8_write(codes, scales, table, k, k, _ints([0, new[0], rows]), _ints(past), max(new), sections=(64,),
                   cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda())
    wc, ws = pool.codes.copy(), pool.scales.copy()
    R.write(wc, ws, pool.table, k64, k64, [0, new[0], rows], past, max(new), [64], None, cos, sin)
    _same_codes(_bits(codes), wc)
    np.testing.assert_array_equal(scales.cpu().numpy(), ws)
