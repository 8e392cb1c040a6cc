"""The pages of an 8-bit KV cache (include/ebrl_kv8_pages.h) against plain lists: forks,
releases, reservations, compaction, alone and in turn; the calls that are refused; a
decoder layer's steps in 8 bits for rollouts that share a prefix."""
import ctypes
import random

import pytest
import torch

from paper_2609_27547_amd import ebrl as E

gpu = pytest.mark.gpu
PAGE = E.KV8_PAGE


# ------------------------------------------------------------ no GPU needed --

def _pool(**kw):
    p = E.Kv8Pool(codes=4096, scales=8192, block_table=12288, refs=16384, layer_codes=1 << 20, layer_scales=1 << 10,
                  layers=2, num_blocks=8, table_rows=2, table_stride=4, kv_heads=2, head_dim=64)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _fork(pool, src=4096, dst=4096, length=4096, n=2):
    return E.lib().ebrl_op_kv8_fork(ctypes.byref(pool), src, dst, length, n, None)


def _free(pool, seq=4096, keep=0, n=2):
    return E.lib().ebrl_op_kv8_free(ctypes.byref(pool), seq, keep, n, None)


def _reserve(pool, seq=4096, pos0=4096, count=4096, n=2, most=40, lacking=4096, work=4096, size=1 << 20):
    return E.lib().ebrl_op_kv8_reserve(ctypes.byref(pool), seq, pos0, count, n, most, lacking, work, size, None)


def _compact(pool, table=4096, refs=4096, used=4096, work=4096, size=1 << 20):
    return E.lib().ebrl_op_kv8_compact(ctypes.byref(pool), table, refs, used, work, size, None)


TABLE = [dict(block_table=0), dict(refs=0), dict(refs=2), dict(num_blocks=0), dict(num_blocks=(1 << 30) + 1),
         dict(table_rows=0), dict(table_stride=0), dict(table_stride=1 << 27)]


@pytest.mark.parametrize("bad", TABLE)
def test_tables_are_refused(bad):
    assert _fork(_pool(**bad)) == _free(_pool(**bad)) == _reserve(_pool(**bad)) == _compact(_pool(**bad)) == -1


@pytest.mark.parametrize("bad", [
    dict(codes=0), dict(codes=4104), dict(scales=0), dict(scales=2), dict(layers=0), dict(layers=65536), dict(kv_heads=0),
    dict(kv_heads=(1 << 17) + 1), dict(head_dim=32), dict(layer_codes=8), dict(layer_codes=-16), dict(layer_scales=-1)])
def test_pools_are_refused(bad):
    assert _reserve(_pool(**bad)) == _compact(_pool(**bad)) == -1


def test_numbers_are_refused():
    p = _pool()
    for kw in (dict(n=-1), dict(n=65537), dict(src=0), dict(dst=0), dict(length=0)):
        assert _fork(p, **kw) == -1
    for kw in (dict(n=-1), dict(n=65537), dict(seq=0)):
        assert _free(p, **kw) == -1
    need = E.lib().ebrl_op_kv8_reserve_workspace(ctypes.byref(p), 2, 40)
    assert 0 < need < 1 << 12
    for kw in (dict(n=-1), dict(n=65537), dict(most=-1), dict(seq=0), dict(pos0=0), dict(count=0), dict(lacking=0), dict(lacking=2),
               dict(work=0), dict(work=4104), dict(size=need - 1)):
        assert _reserve(p, **kw) == -1
    need = E.lib().ebrl_op_kv8_compact_workspace(ctypes.byref(p))
    for kw in (dict(table=0), dict(refs=0), dict(used=0), dict(table=2), dict(refs=1), dict(used=6), dict(work=0), dict(work=8), dict(size=need - 1)):
        assert _compact(p, **kw) == -1
    many = _pool(table_stride=1 << 20, num_blocks=1 << 20)
    assert E.lib().ebrl_op_kv8_reserve_workspace(ctypes.byref(many), 65536, 1 << 30) == -1
    wide = _pool(layers=60000, kv_heads=1 << 10, layer_codes=1 << 30)
    assert _reserve(wide, n=2000, size=1 << 40) == -1
    assert _fork(p, n=0) == _free(p, n=0) == 0 and E.lib().ebrl_op_kv8_reserve_workspace(ctypes.byref(p), 0, 0) >= 0


def test_sizes_that_get_a_workspace_are_taken():
    """What the host refuses for size alone, the workspace's call refuses too.  The calls get a workspace of no bytes,
    so none of them goes on to the GPU."""
    for kw in (dict(num_blocks=1 << 30, kv_heads=1 << 17, head_dim=128), dict(num_blocks=1 << 21, kv_heads=1 << 17),
               dict(num_blocks=1 << 30, kv_heads=1), dict(num_blocks=(1 << 30) + 1), dict(table_stride=1 << 27)):
        p = _pool(**kw)
        need = E.lib().ebrl_op_kv8_compact_workspace(ctypes.byref(p))
        pieces = -(-2 * p.kv_heads * PAGE * p.head_dim // 16384)
        ok = p.num_blocks <= 1 << 30 and p.table_stride < 1 << 27 and p.num_blocks // 2 * pieces <= 1 << 30
        assert (need > 0) == ok and (ok or need == -1)
    for n, most, kw in ((18000, 1, dict(layers=60, kv_heads=32, head_dim=128)), (65536, 1, dict(layers=8, kv_heads=512, head_dim=128)),
                        (65536, 1, dict(layers=9, kv_heads=512, head_dim=128)), (65536, 1, dict(layers=1, kv_heads=512, head_dim=128)),
                        (65536, 1, dict(layers=65535, kv_heads=1)), (2000, 40, dict(layers=60000, kv_heads=1 << 10)),
                        (1, 1, dict(layers=65535, kv_heads=1 << 17, head_dim=128)), (65537, 1, {}), (65536, 0, {}), (0, 0, {}),
                        (65536, 1 << 30, dict(table_stride=1 << 20))):
        p = _pool(**kw)
        need = E.lib().ebrl_op_kv8_reserve_workspace(ctypes.byref(p), n, most)
        pages = min((most + 30) // 16, p.table_stride)
        pieces = -(-2 * p.kv_heads * PAGE * p.head_dim // 16384)
        ok = n <= 65536 and n * pages <= 1 << 30 and n * pieces * -(-p.layers // 8) <= 1 << 23
        assert (need > 0) == ok and (ok or need == -1)
        assert _reserve(p, n=n, most=most, size=0) == -1


def test_binding_refuses():
    codes, scales = E.kv8_alloc(4, 2, 64, device="cpu")
    table, refs = torch.full((2, 3), -1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731

    def refused(f, *a, **kw):
        with pytest.raises(E.EbrlError):
            f(*a, **kw)
    one = i32(0)
    for t, r in ((table, refs), (table.long(), refs), (table[0], refs), (table, refs.long()), (table, refs[::2])):
        refused(E.op_kv8_fork, t, r, one, i32(1), one)           # the first: not on a GPU
        refused(E.op_kv8_free, t, r, one)
    refused(E.op_kv8_fork, table, refs, one, i32(0, 1), one)
    refused(E.op_kv8_fork, table, refs, one.long(), one, one)
    refused(E.op_kv8_free, table, refs, one, i32(1, 2))
    for c, s, t in ((codes, scales, table), (codes.float(), scales, table), (codes[:3], scales[:3], table),
                    (codes, scales.double(), table), (codes, scales[:, :1], table), (codes[:, :1], scales[:, :1], table),
                    (codes[None].expand(2, -1, -1, -1, -1), scales, table)):
        refused(E.op_kv8_reserve, c, s, t, refs, one, one, one, 4, one)
        refused(E.op_kv8_compact, c, s, t, refs, t, refs, one)
    refused(E.op_kv8_reserve, codes, scales, table, refs, one, one, one, -1, one)
    refused(E.op_kv8_reserve, codes, scales, table, refs, one, one, one, 1 << 31, one)
    refused(E.op_kv8_reserve, codes, scales, table, refs, one, one, one, 4, i32(0, 0))
    refused(E.op_kv8_reserve, codes, scales, table, refs, one, one, one, 4, one, stream=0)
    refused(E.op_kv8_compact, codes, scales, table, refs, table[:1], refs, one)
    refused(E.op_kv8_compact, codes, scales, table, refs, table, refs.long(), one)
    refused(E.kv8_reserve_workspace, codes, table, -1, 3)
    refused(E.kv8_reserve_workspace, codes, table, 70000, 3)
    refused(E.kv8_compact_workspace, codes[0], table)


class _Elsewhere(torch.Tensor):
    """A tensor that says it is on another device."""

    def get_device(self):
        return 1


def _elsewhere(t):
    return t.as_subclass(_Elsewhere)


def _table_calls():
    """(message, function, arguments): each call is refused by the check that the message is of."""
    table, refs = torch.full((2, 3), -1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    one, two = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    fork, free = dict(src=one, dst=one, length=one), dict(seq=one)
    pool = dict(block_table=table, refs=refs)
    for f, kw in ((E.op_kv8_fork, fork), (E.op_kv8_free, free), (E.op_kv8_free, free | dict(keep=one))):
        yield "not on a GPU", f, pool | kw
        for t in (refs.long(), refs[::2], refs[None]):
            yield "refs are contiguous int32", f, pool | kw | dict(refs=t)
        for t in (table.long(), table[0], table[:, ::2], table.t(), _elsewhere(table)):
            yield "block_table is contiguous int32", f, pool | kw | dict(block_table=t)
        for name in kw:
            if name in ("dst", "seq") and len(kw) > 1:      # (the one that says how many rows there are)
                other = "src" if name == "dst" else "keep"
                yield f"{other} is 2 contiguous int32", f, pool | kw | {name: two}
            else:
                yield f"{name} is 1 contiguous int32" if len(kw) > 1 else "not on a GPU", f, pool | kw | {name: two}
            for t in (one.long(), _elsewhere(one)):
                yield f"{name} is 1 contiguous int32", f, pool | kw | {name: t}
        name = list(kw)[0]
        spread = torch.zeros(6, dtype=torch.int32)[::3]
        yield f"{name} is 2 contiguous int32", f, pool | {k: two for k in kw} | {name: spread}


def _pool_calls():
    codes, scales = E.kv8_alloc(4, 2, 64, device="cpu")
    table, refs = torch.full((2, 3), -1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    one, two = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    work = torch.zeros(4096, dtype=torch.uint8)
    raw = codes.view(torch.uint8)
    many, many_scales = raw[None].repeat(3, 1, 1, 1, 1), scales[None].repeat(3, 1, 1, 1)
    pool = dict(codes=codes, scales=scales, block_table=table, refs=refs)
    reserve = dict(seq=one, pos0=one, count=one, max_count=4, lacking=one)
    compact = dict(new_table=table, new_refs=refs, used=one)
    for f, kw, ints in ((E.op_kv8_reserve, reserve, ["pos0", "count", "lacking"]), (E.op_kv8_compact, compact, ["used"])):
        gap = raw.new_zeros((3, 6, 2, 2, 1024))[:, :4]
        for more in ({}, dict(workspace=work), dict(workspace=work, stream=0), dict(codes=raw), dict(codes=many, scales=many_scales),
                     dict(codes=gap, scales=many_scales)):
            yield "not on a GPU", f, pool | kw | more
        yield "refs are contiguous int32", f, pool | kw | dict(refs=refs.long())
        yield "block_table is contiguous int32", f, pool | kw | dict(block_table=table[0])
        for t in (codes.float(), codes[0], raw[:, :1], raw[..., :1000], raw[..., :0], many[None], many[:0]):
            yield "codes are float8_e4m3fn or bytes", f, pool | kw | dict(codes=t)
        for t in (raw[:3], raw.transpose(1, 2), raw[:, :, :1], _elsewhere(raw), many[:, :, :, :1], raw.new_zeros((4, 2, 2, 2048))[..., ::2]):
            yield "codes of a layer are contiguous", f, pool | kw | dict(codes=t, scales=many_scales if t.dim() == 5 else scales)
        for t in (scales.double(), scales[:3], scales[:, :1], scales[None], scales.new_ones((4, 2, 4))[..., ::2], _elsewhere(scales)):
            yield "scales are float32", f, pool | kw | dict(scales=t)
        yield "scales are float32", f, pool | kw | dict(codes=many, scales=many_scales[:2])
        yield "scales are float32", f, pool | kw | dict(codes=many, scales=many_scales.transpose(2, 3))
        for name in ints:
            for t in (two, one.long(), _elsewhere(one)):
                yield f"{name} is 1 contiguous int32", f, pool | kw | {name: t}
        yield "explicit stream needs a workspace", f, pool | kw | dict(stream=0)
        for t in (torch.zeros((64, 64))[:, ::2], _elsewhere(work)):
            yield "workspace is contiguous and where", f, pool | kw | dict(workspace=t)
    yield "pos0 is 2 contiguous int32", E.op_kv8_reserve, pool | reserve | dict(seq=two)
    yield "seq is 1 contiguous int32", E.op_kv8_reserve, pool | reserve | dict(seq=one.long())
    for n in (-1, 1 << 31):
        yield f"max_count {n}", E.op_kv8_reserve, pool | reserve | dict(max_count=n)
    for name, t in (("new_table", table[:1]), ("new_refs", refs[:3])):
        yield "have the shapes of block_table and refs", E.op_kv8_compact, pool | compact | {name: t}
    for name, t in (("new_table", table.long()), ("new_table", torch.zeros((3, 2), dtype=torch.int32).t()),
                    ("new_table", _elsewhere(table)), ("new_refs", refs.long()), ("new_refs", _elsewhere(refs))):
        yield f"{name} is [0-9]+ contiguous int32", E.op_kv8_compact, pool | compact | {name: t}
    for sizes in ((-1, 3), (1, -1), (1 << 31, 3), (1, 1 << 31)):
        yield "ebrl_op_kv8_reserve_workspace: ", E.kv8_reserve_workspace, dict(codes=codes, block_table=table, n=sizes[0],
                                                                              max_count=sizes[1])
    for f, kw in ((E.kv8_reserve_workspace, dict(n=1, max_count=1)), (E.kv8_compact_workspace, {})):
        yield r"block_table is \[sequences, pages\]", f, dict(codes=codes, block_table=table[0]) | kw
        yield "codes are float8_e4m3fn or bytes", f, dict(codes=codes[0], block_table=table) | kw


@pytest.mark.parametrize("calls", [_table_calls, _pool_calls], ids=["tables", "pools"])
def test_binding_refuses_each_argument(calls):
    """By the check that is meant: calls that are right get as far as the one that asks for a GPU."""
    for message, f, kw in calls():
        with pytest.raises(E.EbrlError, match=message):
            f(**kw)


@pytest.mark.parametrize("n", [65537, (1 << 32) + 1])
def test_more_rows_than_a_call_takes(n):
    """Refused for their number, also where its low 32 bits are a small one (tensors without memory)."""
    table, refs, ids, one = (torch.empty(s, dtype=torch.int32, device="meta") for s in ((2, 3), (4,), (n,), (1,)))
    codes = torch.empty((4, 2, 2, 1024), dtype=torch.uint8, device="meta")
    scales = torch.empty((4, 2, 2), device="meta")
    for call in (lambda: E.op_kv8_fork(table, refs, ids, ids, ids), lambda: E.op_kv8_free(table, refs, ids),
                 lambda: E.op_kv8_reserve(codes, scales, table, refs, ids, ids, ids, 1, one, workspace=one)):
        with pytest.raises(E.EbrlError, match="at most 65536 rows"):
            call()


# ------------------------------------------------------------- plain lists --

class Lists:
    """A pool in plain lists; a page's content is a number for each layer and group, in all its bytes."""

    def __init__(self, layers, num, rows, stride, heads, hd, gap=0):
        self.layers, self.num, self.rows, self.stride, self.heads, self.hd = layers, num, rows, stride, heads, hd
        self.table = [[-1] * stride for _ in range(rows)]
        self.refs = [0] * num
        self.store = torch.zeros((layers, num + gap, 2, heads, PAGE * hd), dtype=torch.uint8, device="cuda")
        self.codes = self.store[:, :num]
        self.scales = torch.zeros((layers, num + gap, 2, heads), device="cuda")[:, :num]
        self.content = list(range(num))                # what each page holds
        for lo in range(0, num, 4096):
            self.codes[:, lo:lo + 4096], self.scales[:, lo:lo + 4096] = self._pattern(
                torch.arange(lo, min(num, lo + 4096), device="cuda")[:, None, None])
        self.d_table = torch.full((rows, stride), -1, dtype=torch.int32, device="cuda")
        self.d_refs = torch.zeros(num, dtype=torch.int32, device="cuda")
        self.lacking = torch.full((1,), 99, dtype=torch.int32, device="cuda")

    def _pattern(self, v):
        n = self.layers * 2 * self.heads
        which = torch.arange(n, device="cuda").reshape(self.layers, 1, 2, self.heads)
        at = torch.arange(PAGE * self.hd, device="cuda")
        c, s = (v * 31 + which) * 7, v * 1000 + which
        return ((c[..., None] + at * ((v % 5 + 1)[..., None])) % 251).to(torch.uint8), s.float()

    def fill(self, p, v):
        self.codes[:, p:p + 1], self.scales[:, p:p + 1] = self._pattern(torch.tensor([v], device="cuda")[:, None, None])
        self.content[p] = v

    def check(self):
        torch.cuda.synchronize()
        assert self.d_table.tolist() == self.table
        assert self.d_refs.tolist() == self.refs
        for lo in range(0, self.num, 4096):
            c, s = self._pattern(torch.tensor(self.content[lo:lo + 4096], device="cuda")[:, None, None])
            same = (self.codes[:, lo:lo + 4096] == c).flatten(2).all(2) & (self.scales[:, lo:lo + 4096] == s).flatten(2).all(2)
            assert same.all(), f"pages {(lo + torch.nonzero(~same.all(0)).flatten()).tolist()[:9]}"
        # nothing behind a layer's last page was touched
        assert (self.store[:, self.num:] == 0).all()

    def held(self, tokens):
        return min((min(max(tokens, 0), self.stride * PAGE) + PAGE - 1) // PAGE, self.stride)

    def page(self, p):
        return 0 <= p < self.num

    def fork(self, src, dst, length):
        named = set(dst)
        for i, (s, d, t) in enumerate(zip(src, dst, length)):
            if not 0 <= s < self.rows or not 0 <= d < self.rows or s in named or d in dst[:i]:
                continue
            new = [p if j < self.held(t) and self.page(p) else -1 for j, p in enumerate(self.table[s])]
            for p in self.table[d]:
                if self.page(p):
                    self.refs[p] -= 1
            for p in new:
                if p >= 0:
                    self.refs[p] += 1
            self.table[d] = new
        E.op_kv8_fork(self.d_table, self.d_refs, _i32(src), _i32(dst), _i32(length))

    def free(self, seq, keep=None):
        for i, s in enumerate(seq):
            if 0 <= s < self.rows:
                for j in range(self.held(keep[i]) if keep else 0, self.stride):
                    if self.page(self.table[s][j]):
                        self.refs[self.table[s][j]] -= 1
                    self.table[s][j] = -1
        E.op_kv8_free(self.d_table, self.d_refs, _i32(seq), None if keep is None else _i32(keep))

    def reserve(self, seq, pos0, count, most, **kw):
        before, free = list(self.refs), [p for p, r in enumerate(self.refs) if r <= 0]
        todo = []
        for i, (s, pos, n) in enumerate(zip(seq, pos0, count)):
            if not 0 <= s < self.rows or s in seq[:i]:
                continue
            pos = max(pos, 0)
            end = min(pos + min(max(n, 0), most), self.stride * PAGE)
            for j in range(pos // PAGE, (end + PAGE - 1) // PAGE if end > pos else 0):
                p = self.table[s][j]
                if not self.page(p) or before[p] > 1:
                    todo.append((s, j, p, j == pos // PAGE and pos % PAGE > 0))
        short = max(0, len(todo) - len(free))
        if not short:
            for (s, j, p, copy), q in zip(todo, free):
                self.table[s][j], self.refs[q] = q, 1
                if self.page(p):
                    self.refs[p] -= 1
                    if copy:
                        self.content[q] = self.content[p]
        E.op_kv8_reserve(self.codes, self.scales, self.d_table, self.d_refs, _i32(seq), _i32(pos0), _i32(count), most,
                         self.lacking, **kw)
        assert self.lacking.item() == short
        return short

    def compact(self, apart=False, **kw):
        end = sum(r > 0 for r in self.refs)
        holes = [p for p in range(end) if self.refs[p] <= 0]
        to = dict(zip([p for p in range(end, self.num) if self.refs[p] > 0], holes))
        for a, b in to.items():
            self.refs[b], self.content[b] = self.refs[a], self.content[a]
        self.refs = [r if p < end else 0 for p, r in enumerate(self.refs)]
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        used = torch.full((1,), -5, dtype=torch.int32, device="cuda")
        table, refs = (torch.full_like(self.d_table, 77), torch.full_like(self.d_refs, 77)) if apart else \
            (self.d_table, self.d_refs)
        E.op_kv8_compact(self.codes, self.scales, self.d_table, self.d_refs, table, refs, used, **kw)
        self.d_table, self.d_refs = table, refs
        assert used.item() == end


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


SIZES = [(1, 40, 6, 8, 1, 64, 0), (3, 60, 10, 12, 4, 128, 2), (2, 500, 20, 40, 2, 64, 0), (1, 9000, 12, 700, 1, 64, 1),
         (5, 30, 4, 300, 16, 128, 0), (2, 4097, 9, 5, 1, 64, 0),
         (1, 65536, 5, 9000, 1, 64, 0), (1, 70001, 5, 9000, 1, 64, 3), (2, 300, 70, 60, 17, 128, 0)]


@gpu
@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("seed", [0, 1])
def test_calls_in_turn(sizes, seed):
    """Calls of every kind, one after the other, with numbers outside the table among theirs."""
    r = random.Random(seed * 100 + sizes[1])
    p = Lists(*sizes)
    most = p.stride * PAGE
    for step in range(30):
        n = r.randrange(1, p.rows + 3)
        rows = [r.randrange(-1, p.rows + 1) for _ in range(n)]
        what = r.choice(["fork", "free", "reserve", "reserve", "compact"])
        if what == "fork":
            p.fork([r.randrange(-1, p.rows + 1) for _ in range(n)], rows, [r.randrange(-5, most + 40) for _ in range(n)])
        elif what == "free":
            p.free(rows, r.choice([None, [r.randrange(-5, most + 40) for _ in range(n)]]))
        elif what == "reserve":
            cap = max(1, min(most, p.num * PAGE // (2 * n)))
            p.reserve(rows, [r.randrange(-3, cap + 20) for _ in range(n)], [r.randrange(-3, cap) for _ in range(n)],
                      r.choice([0, 1, cap // 2, cap]))
        else:
            p.compact(apart=r.random() < 0.5)
        if step % 6 == 5 or p.num < 1000:
            p.check()
        for q in range(0, p.num, 1 + p.num // 50):            # new contents from time to time
            if p.refs[q] and r.random() < 0.1:
                p.fill(q, r.randrange(1 << 16))
    p.check()
    assert sum(x for x in p.refs) == sum(q >= 0 for row in p.table for q in row)


@gpu
@pytest.mark.parametrize("rows,num", [(1024, 4000), (1025, 4000), (1300, 5000), (1500, 70000)])
def test_many_rows(rows, num):
    r = random.Random(rows)
    p = Lists(1, num, rows, 3, 1, 64)
    first = [r.randrange(-2, rows + 2) for _ in range(rows - 200)] + [5] * 200
    p.reserve(first, [0] * rows, [r.randrange(0, 49) for _ in range(rows)], 48)
    src = [i for i in range(100) if p.table[i][0] >= 0]
    dst = [r.randrange(100, rows) for _ in src]
    p.fork(src, dst, [r.randrange(1, 49) for _ in src])
    p.check()
    order = r.sample(range(rows), rows)
    p.reserve(order, [r.randrange(0, 40) for _ in order], [r.randrange(0, 20) for _ in order], 20)
    p.check()
    p.free(r.sample(range(rows), rows // 2))
    p.compact()
    p.check()
    assert sum(p.refs) == sum(q >= 0 for row in p.table for q in row)


@gpu
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_refs_of_any_alignment(shift):
    """refs at any element of a larger tensor."""
    p = Lists(1, 100, 6, 20, 1, 64)
    p.d_refs = torch.zeros(100 + shift, dtype=torch.int32, device="cuda")[shift:]
    p.reserve([0, 1, 2], [0, 0, 0], [300, 200, 77], 320)
    p.fork([0, 1], [3, 4], [300, 133])
    p.reserve([3, 4], [300, 133], [9, 9], 9)
    p.free([0, 2])
    p.compact()
    p.check()


@gpu
def test_branches_write_to_pages_of_their_own():
    p = Lists(2, 40, 6, 6, 2, 128)
    p.reserve([0], [0], [40], 40)                             # pages 0, 1, 2; eight tokens in the last
    p.fork([0, 0, 0], [1, 2, 3], [40, 32, 33])
    assert p.refs[:3] == [4, 4, 3]
    p.reserve([1, 2, 3, 0], [40, 32, 33, 40], [1, 20, 1, 0], 20)
    # row 1: a copy of its last page; row 2: no page yet, so no copy; row 3: a copy; row 0: nothing to write
    assert p.table[1][:3] == [0, 1, 3] and p.table[2][:4] == [0, 1, 4, 5] and p.table[3][:3] == [0, 1, 6]
    assert p.content[3] == p.content[6] == p.content[2] and p.content[4] == 4 and p.refs[2] == 1
    p.check()
    p.reserve([0], [40], [1], 1)                              # now its own
    assert p.table[0][:3] == [0, 1, 2]
    p.free([1, 2, 3], [0, 16, 48])
    assert p.table[2][0] == 0 and p.refs[:3] == [3, 2, 1]
    p.check()
    p.compact()
    p.check()


@gpu
def test_pages_that_are_lacking():
    """One page too few: nothing changes, and the number is told; then exactly enough."""
    p = Lists(2, 9, 5, 6, 1, 64)
    p.reserve([0], [0], [50], 50)
    p.fork([0, 0, 0], [1, 2, 3], [50, 50, 50])
    assert p.reserve([1, 2, 3, 4], [50, 50, 50, 0], [1, 1, 1, 48], 48) == 1
    p.check()
    assert p.reserve([1, 2, 3, 4], [50, 50, 50, 0], [1, 1, 1, 30], 48) == 0
    p.check()
    assert p.reserve([0], [95], [1], 48) == 1 and p.reserve([0], [96], [1], 48) == 0 and p.reserve([], [], [], 3) == 0
    p.check()


@gpu
def test_pools_without_a_page_in_use_and_with_all():
    for num in (1, 2, 4096, 5000):
        p = Lists(1, num, 3, num + 1, 1, 64)
        p.compact()
        p.free([0, 1, 2])
        p.check()
        p.reserve([2], [0], [num * PAGE], num * PAGE)
        p.compact(apart=True)
        assert p.table[2] == list(range(num)) + [-1]
        assert p.reserve([1], [0], [1], 1) == 1
        p.free([2], [16])
        p.compact()
        p.check()


@gpu
def test_entries_that_hold_no_page_and_refs_below_zero():
    """Ids outside the pool in a table are no pages; negative refs are free pages; nothing is read past them."""
    p = Lists(1, 20, 3, 4, 1, 64)
    p.table = [[25, -7, 3, 1 << 30], [-1, 4, 19, -1 << 31], [5, 5, 5, 6]]
    p.refs = [0, -3, 0, 1, 1, 3, 1] + [0] * 12 + [1]
    p.d_table.copy_(_i32(p.table))
    p.d_refs.copy_(_i32(p.refs))
    p.compact(apart=True)
    p.check()
    p.fork([0], [1], [64])
    p.check()
    p.reserve([0, 2], [0, 0], [64, 64], 64)
    p.check()


@gpu
def test_captured_calls_are_replayed():
    """Release, fork and reservation in a graph, with eager work on the same pool between the replays."""
    p = Lists(3, 200, 12, 10, 2, 64)
    p.reserve([0, 1], [0, 0], [90, 77], 90)
    src, dst, length = [0, 1, 0, 1], [2, 3, 4, 5], [90, 77, 85, 64]
    t = [_i32(x) for x in (src, dst, length, [7] * 4)]
    work = E.kv8_reserve_workspace(p.codes, p.d_table, 4, 7)
    side = torch.cuda.Stream()

    def step():
        E.op_kv8_free(p.d_table, p.d_refs, t[1])
        E.op_kv8_fork(p.d_table, p.d_refs, t[0], t[1], t[2])
        E.op_kv8_reserve(p.codes, p.scales, p.d_table, p.d_refs, t[1], t[2], t[3], 7, p.lacking, workspace=work)

    def plain():
        p.free(dst)
        p.fork(src, dst, length)
        p.reserve(dst, length, [7] * 4, 7)
    plain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(4):
        p.reserve([6 + i], [0], [20 + i], 40)                 # other rows take pages meanwhile
        if i == 2:
            p.compact()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        after = (p.d_table.clone(), p.d_refs.clone(), p.codes.clone())
        plain()                                               # the same again on what the replay left
        assert torch.equal(after[0], p.d_table) and torch.equal(after[1], p.d_refs) and torch.equal(after[2], p.codes)
        p.check()


@gpu
@pytest.mark.parametrize("rows,layers,heads", [(18000, 60, 32), (65536, 20, 128), (4000, 300, 64)])
def test_reservations_of_many_workgroups(rows, layers, heads):
    """Rows x pieces of a page x layers past 2^23, which eight layers a workgroup bring below it: many rows of which a
    few need a page; every layer of a copy is there."""
    num, hd = 6, 128
    codes = torch.zeros((layers, num, 2, heads, PAGE * hd), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((layers, num, 2, heads), device="cuda")
    codes[:, 1] = (torch.arange(layers, device="cuda") % 251 + 1).to(torch.uint8)[:, None, None, None]
    codes[:, 1, 1, heads - 1, -1] = 255
    scales[:, 1] = torch.arange(1, layers + 1, device="cuda")[:, None, None]
    table = torch.full((rows, 2), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(num, dtype=torch.int32, device="cuda")
    sharers = [0, rows // 2, rows - 1]
    table[sharers, 0] = 1
    refs[1] = 3
    count = torch.zeros(rows, dtype=torch.int32, device="cuda")
    count[[rows // 2, rows - 1, rows // 3]] = 1
    lacking = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    E.op_kv8_reserve(codes, scales, table, refs, torch.arange(rows, dtype=torch.int32, device="cuda"),
                     torch.full((rows,), 7, dtype=torch.int32, device="cuda"), count, 1, lacking)
    # in the rows' order: a third of them down a page of its own, then two copies
    assert lacking.item() == 0 and refs.tolist() == [1, 1, 1, 1, 0, 0]
    want = torch.full_like(table, -1)
    want[rows // 3, 0], want[rows // 2, 0], want[rows - 1, 0], want[0, 0] = 0, 2, 3, 1
    assert torch.equal(table, want)
    for p in (2, 3):
        assert torch.equal(codes[:, p], codes[:, 1]) and torch.equal(scales[:, p], scales[:, 1])
    assert not codes[:, [0, 4, 5]].any() and not scales[:, [0, 4, 5]].any()


@gpu
def test_pool_past_four_gigabytes():
    """Layers more than 4 GiB apart, ids whose bytes pass 32 bits."""
    num = 40000
    store = torch.zeros((2, num, 2, 32, PAGE * 128), dtype=torch.uint8, device="cuda")       # 5.2 GB a layer
    scales = torch.zeros((2, num, 2, 32), device="cuda")
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    refs = torch.ones(num, dtype=torch.int32, device="cuda")
    refs[num - 1] = refs[num - 3] = 0
    table[0, 0] = num - 2
    refs[num - 2] = 2
    store[:, num - 2] = 113
    store[1, num - 2, 1] = 7
    scales[:, num - 2] = 0.5
    lacking = torch.zeros(1, dtype=torch.int32, device="cuda")
    E.op_kv8_reserve(store, scales, table, refs, _i32([0]), _i32([5]), _i32([1]), 1, lacking)
    assert table[0].tolist() == [num - 3, -1, -1, -1] and lacking.item() == 0
    assert torch.equal(store[:, num - 3], store[:, num - 2]) and (scales[:, num - 3] == 0.5).all()
    assert (store[:, num - 4] == 0).all() and (store[:, num - 1] == 0).all()


# -------------------------------------------------- a layer's steps together --

@gpu
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (4, 4, 128)])
def test_decoder_layer_steps_for_rollouts_of_one_prefix(hq, hkv, hd):
    """A prefix is written once; branches are forked from it and take three steps of a layer in 8 bits: pages,
    pre-norm to codes, projection, rotary write, attention, output projection onto the residual stream.  Every
    branch's rows are, bit for bit, those of a sequence of its own that wrote the same prefix itself."""
    g = torch.Generator().manual_seed(3)
    d, prefix, branches, steps = hq * hd, 53, 5, 3
    wide = (hq + 2 * hkv) * hd
    wqkv, sqkv = E.i8_alloc(wide, d)
    E.op_i8_quant((torch.randn((wide, d), generator=g) * d ** -0.5).cuda(), wqkv, sqkv)
    wo, so = E.i8_alloc(d, d)
    E.op_i8_quant((torch.randn((d, d), generator=g) * d ** -0.5).cuda(), wo, so)
    ang = torch.arange(128).double()[:, None] * 10000.0 ** (-torch.arange(hd // 2).double() * 2 / hd)
    cos, sin = ang.cos().float().cuda(), ang.sin().float().cuda()
    start_x = torch.randn((prefix, d), generator=g).cuda()
    step_x = torch.randn((steps, branches, d), generator=g).cuda()

    def layer(x, cache, table, refs, seq, pos0, count):
        """x [n * count, d]: count new tokens of each row in seq."""
        n = len(seq)
        codes, scales = cache
        lacking = torch.zeros(1, dtype=torch.int32, device="cuda")
        E.op_kv8_reserve(codes, scales, table, refs, _i32(seq), _i32(pos0), _i32([count] * n), count, lacking)
        assert lacking.item() == 0
        a, sa = E.i8_alloc(len(x), d)
        E.op_i8_quant(x, a, sa, norm_eps=1e-6)
        qkv = torch.empty((len(x), wide), dtype=torch.bfloat16, device="cuda")
        E.op_i8_gemm(a, sa, wqkv, sqkv, qkv)
        q, k, v = qkv.split([hq * hd, hkv * hd, hkv * hd], 1)
        rows = _i32([i * count for i in range(n + 1)])
        turned, o = torch.empty_like(x, dtype=torch.bfloat16), torch.empty_like(x, dtype=torch.bfloat16)
        E.op_kv8_write(codes, scales, table, k, v, rows, _i32(pos0), count, q=q, q_out=turned, sections=(hd // 2,),
                       cos=cos, sin=sin, seq=_i32(seq))
        E.op_kv8_attn(codes, scales, table, turned, o, rows, _i32([p + count for p in pos0]), count, 128, seq=_i32(seq))
        E.op_i8_quant(o, a, sa)
        y = x.clone()
        E.op_i8_gemm(a, sa, wo, so, y, residual=y)
        return y

    def new_pool():
        return E.kv8_alloc(64, hkv, hd), torch.full((branches + 1, 8), -1, dtype=torch.int32, device="cuda"), \
            torch.zeros(64, dtype=torch.int32, device="cuda")
    shared, table, refs = new_pool()
    layer(start_x, shared, table, refs, [0], [0], prefix)
    rows = list(range(1, branches + 1))
    E.op_kv8_fork(table, refs, _i32([0] * branches), _i32(rows), _i32([prefix] * branches))
    assert (refs > 0).sum().item() == 4
    alone, table2, refs2 = new_pool()
    for r in rows:
        layer(start_x, alone, table2, refs2, [r], [0], prefix)
    for t in range(steps):
        y = layer(step_x[t], shared, table, refs, rows, [prefix + t] * branches, 1)
        z = layer(step_x[t], alone, table2, refs2, rows, [prefix + t] * branches, 1)
        assert torch.equal(y, z) and y.isfinite().all()
    assert (refs > 0).sum().item() == 4 + branches and (refs2 > 0).sum().item() == 4 * branches
    # the prefix kept its own last page; two rollouts end, the pool closes up, the others go on
    E.op_kv8_free(table, refs, _i32([0, 2]))
    used = torch.zeros(1, dtype=torch.int32, device="cuda")
    E.op_kv8_compact(*shared, table, refs, table, refs, used)
    assert used.item() == 3 + 4 and table.max().item() == used.item() - 1
    left = [r for r in rows if r != 2]
    x = torch.randn((len(left), d), generator=g).cuda()
    assert torch.equal(layer(x, shared, table, refs, left, [prefix + steps] * 4, 1),
                       layer(x, alone, table2, refs2, left, [prefix + steps] * 4, 1))
