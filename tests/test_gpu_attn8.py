"""Attention over the paged 8-bit cache against the 64-bit oracle.

Tolerances, for a row that sees n keys, with p the exact weights and A_d = sum p |v_d|:
  - a score is a sum of dim exact products in fp32, times two numbers and less a third:
    (dim + 8) 2^-24 of scale * sum |q k| and 4 * 2^-24 of the largest |score|.  A weight is off by that (e, the
    largest over the keys) and by 2^-21 (the power of two, two products), and so is their sum: 2 e + 2^-20 of A_d;
  - a weight's rounding to parts of bf16: 2^-8 (bf16), 2^-16 (fp16, two parts), 2^-24 (fp32, three);
  - sums of n terms in fp32, in parts that are joined: (n + 16) 2^-24, for the weights' sum too;
  - half a step of the output's type.
"""
import numpy as np
import pytest

from oracle import attn8, q8
from test_gpu_cache8 import HALF, TINY, dtypes, env, typed  # noqa: F401

pytestmark = pytest.mark.gpu

WEIGHT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -16, "float32": 2.0 ** -24}


class Problem:
    """A cache of random codes where tokens are and of NaNs where none are, lists, queries."""

    def __init__(self, torch, L, rng, new, lengths, *, heads=2, group=2, dim=64, page=16, fmt=q8.E4M3, kind=q8.POW2,
                 name="bfloat16", first=0, extra=2, bad=(), cols=None, peaked=1.0, behind=2):
        f, sk = dtypes(torch)
        self.torch, self.L, self.fmt, self.kind, self.name = torch, L, fmt, kind, name
        seqs = len(new)
        width = cols or max(1, max((-(-n // page) for n in lengths), default=1))
        pages = int(sum(-(-n // page) for n in lengths)) + extra
        order = rng.permutation(pages)
        table = rng.integers(0, pages, (seqs, width)).astype(np.int32)
        live = np.zeros((pages, page), bool)
        at = 0
        for b, n in enumerate(lengths):
            m = -(-n // page)
            table[b, :m] = order[at:at + m]
            for c in range(m):
                live[table[b, c], : n - c * page] = True
            at += m
        for b, col, number in bad:
            table[b, col] = number
        self.starts = (first + np.concatenate([[0], np.cumsum(new)])).astype(np.int32)
        self.lengths, self.table, self.page, self.pages = np.asarray(lengths, np.int32), table, page, pages
        self.tokens = int(self.starts[-1]) + behind
        self.heads, self.group, self.dim = heads, group, dim
        codes, scales = [], []
        for _ in range(2):
            c = q8.encode(rng.standard_normal((pages, heads, page, dim)) * q8.MOST[fmt] / 4, fmt)
            c[~live[:, None, :].repeat(heads, 1)] = 0x7F                                 # NaN of both formats
            codes.append(c)
            s = np.exp2(rng.integers(-10, -7, (pages, heads, page)).astype(np.float64)) * (448.0 / q8.MOST[fmt])
            if kind == q8.F32:
                s = (s * rng.uniform(0.5, 1.0, s.shape)).astype(np.float32).astype(np.float64)
            s[~live[:, None, :].repeat(heads, 1)] = np.nan
            scales.append(s)
        self.codes, self.scales = codes, scales
        self.put()
        self.lists = [torch.from_numpy(a).cuda() for a in (self.starts, self.lengths, self.table)]
        self.chunk = L.Chunk(*self.lists)
        self.q, self.eq = typed(torch, peaked * rng.standard_normal((self.tokens, heads * group, dim)), name)

    def put(self):
        torch = self.torch
        f, sk = dtypes(torch)
        k8, v8 = (torch.from_numpy(c).cuda().view(f[self.fmt]) for c in self.codes)
        if self.kind == q8.POW2:
            s = [torch.from_numpy(np.where(np.isnan(s), 255, np.log2(np.nan_to_num(s, nan=1.0)) + 127).astype(np.uint8))
                 .cuda().view(sk[self.kind]) for s in self.scales]
        else:
            s = [torch.from_numpy(s.astype(np.float32)).cuda() for s in self.scales]
        self.cache = self.L.Cache8.of(k8, v8, *s)

    def values(self, which, b, length):
        """(rows [length, heads, dim], which have a place) of a sequence."""
        rows, has = np.zeros((length, self.heads, self.dim)), np.zeros(length, bool)
        for j in range(length):
            page, off = attn8.place(self.table[b], j, self.page, self.pages)
            if page is not None:
                has[j] = True
                rows[j] = q8.decode(self.codes[which][page, :, off], self.fmt) * self.scales[which][page, :, off, None]
        return rows, has

    def row(self, q, k, v, sees, scale):
        """(out, how far from it a row may be, log of the sum, how far that may be) of one row."""
        want, total, room, p = attn8.attend(q, k, v, sees, scale)
        if len(p) == 0:
            return want, 0 * want, total, 0.0
        mags = abs(scale) * (np.abs(k[sees]) @ np.abs(q))
        e = (self.dim + 8) * 2.0 ** -24 * mags.max() + 4 * 2.0 ** -24 * np.abs(scale * (k[sees] @ q)).max()
        add = (len(p) + 16) * 2.0 ** -24
        lim = room * (2 * e + 2.0 ** -20 + WEIGHT[self.name] + 2 * add) + np.abs(want) * HALF[self.name] + TINY[self.name]
        # (2^-8: products of these)
        return want, lim * (1 + 2.0 ** -8), total, e + 2.0 ** -20 + add + 4 * 2.0 ** -24 * abs(total)

    def check(self, out, lse=None, *, scale=None, causal=True, window=0, max_len=0, blank=5.0, rows=None):
        scale = self.dim ** -0.5 if scale is None else scale
        got = out.double().cpu().numpy()
        sums = None if lse is None else lse.double().cpu().numpy()
        mine = np.zeros(self.tokens, bool)
        for b, n in enumerate(self.lengths):
            s0, s1 = self.starts[b], self.starts[b + 1]
            mine[s0:s1] = True
            if s0 == s1:
                continue
            held = len(self.table[b]) * self.page
            length = int(min(n, held, max_len or held))
            (k, has), (v, _) = self.values(0, b, length), self.values(1, b, length)
            j = np.arange(length)
            for t in range(s0, s1):
                pos = int(n) - s1 + t
                sees = has.copy()
                if causal:
                    sees &= j <= pos
                    if window:
                        sees &= j > pos - window
                for h in range(self.eq.shape[1]):
                    if rows is not None and (t, h) not in rows:
                        continue
                    kv = h // self.group
                    q = self.eq[t, h]
                    want, lim, total, off = self.row(q, k[:, kv], v[:, kv], sees, scale)
                    where = f"sequence {b} token {t} head {h}"
                    err = np.abs(got[t, h] - want)
                    assert (err <= lim).all(), (where, float(np.max(err / (lim + 1e-300))))
                    if sums is not None:
                        assert sums[t, h] == total or abs(sums[t, h] - total) <= off, (where, sums[t, h], total, off)
        assert (got[~mine] == blank).all()
        assert sums is None or (sums[~mine] == blank).all()

    def run(self, q=None, **kw):
        torch = self.torch
        q = self.q if q is None else q
        out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device="cuda")
        self.L.ds_attn8(q, self.cache, self.chunk, out, lse, **kw)
        torch.cuda.synchronize()
        return out, lse


# (new tokens, lengths, first token of the call): empty sequences, rows that see nothing, tails of tiles and pages
LISTS = [([1], [1], 0), ([1], [33], 0), ([5, 0, 1, 0], [5, 9, 64, 0], 2), ([3, 2], [1, 2], 1), ([17], [300], 0),
         ([1, 1, 1, 1, 1], [1, 31, 32, 65, 129], 0), ([0, 0], [7, 0], 1), ([150, 1, 3], [150, 40, 70], 0)]


@pytest.mark.parametrize("lists", LISTS, ids=str)
@pytest.mark.parametrize("dim", [16, 64, 80, 128, 144, 256])
@pytest.mark.parametrize("name", ["bfloat16", "float16", "float32"])
def test_attention(env, lists, dim, name):  # noqa: F811
    torch, L = env
    if name == "float32" and dim > 128:
        pytest.skip("refused")
    for i, (heads, group, page, fmt, kind) in enumerate(((1, 1, 16, q8.E4M3, q8.POW2), (2, 3, 48, q8.E5M2, q8.F32),
                                                         (3, 8, 64, q8.E4M3, q8.F32))):
        rng = np.random.default_rng(dim + 17 * i + len(lists[0]))
        p = Problem(torch, L, rng, *lists[:2], first=lists[2], heads=heads, group=group, dim=dim, page=page, fmt=fmt,
                    kind=kind, name=name)
        print(lists, dim, name, i, flush=True)
        p.check(*p.run())


@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
@pytest.mark.parametrize("dim", [48, 64, 80, 128])
@pytest.mark.parametrize("name", ["bfloat16", "float16"])
def test_many_rows(env, dim, name, kind):  # noqa: F811
    """Prompts and chunks: several tiles of rows and of keys, ragged, with and without a window, either sign of
    the scale, and parts of them by split keys."""
    torch, L = env
    for fmt, page, scale, window in ((q8.E4M3, 16, None, 0), (q8.E5M2, 48, -0.2, 0), (q8.E4M3, 64, 0.0, 70)):
        rng = np.random.default_rng(dim + page)
        p = Problem(torch, L, rng, [150, 5, 90], [390, 64, 333], heads=1, group=3, dim=dim, page=page, fmt=fmt, kind=kind,
                    name=name, first=1, bad=[(0, 2, -5)] if page == 48 else ())
        print(dim, name, kind, page, flush=True)
        p.check(*p.run(scale=scale, window=window), scale=scale, window=window)
    p = Problem(torch, L, rng, [70], [9000], heads=1, group=4, dim=dim, page=64, kind=kind, name=name)
    assert L.ds_attn8_work(p.q, p.cache, p.chunk) > 0
    p.check(*p.run(), rows={(t, h) for t in (0, 33, 69) for h in (0, 3)})
    p.check(*p.run(causal=False), causal=False, rows={(t, h) for t in (0, 69) for h in (1,)})


@pytest.mark.parametrize("window", [1, 5, 32, 100])
@pytest.mark.parametrize("lists", [([1, 3], [200, 90], 0), ([90], [90], 0), ([20, 300], [400, 310], 1)], ids=str)
def test_window(env, lists, window):  # noqa: F811
    torch, L = env
    for group, name in ((1, "bfloat16"), (4, "float32")):
        p = Problem(torch, L, np.random.default_rng(window), *lists[:2], first=lists[2], group=group, dim=32, name=name)
        p.check(*p.run(window=window), window=window)


@pytest.mark.parametrize("lists", LISTS, ids=str)
def test_all_keys(env, lists):  # noqa: F811
    """Not causal: every token sees its whole sequence."""
    torch, L = env
    p = Problem(torch, L, np.random.default_rng(1), *lists[:2], first=lists[2], dim=96, group=2)
    p.check(*p.run(causal=False), causal=False)


def test_settings(env):  # noqa: F811
    """Scales of either sign and size, sharp and flat rows, a limit of the lengths."""
    torch, L = env
    for scale, peaked in ((0.0, 1.0), (-0.3, 1.0), (1.0, 4.0), (1e-4, 1.0), (0.125, 0.0)):
        p = Problem(torch, L, np.random.default_rng(2), [3, 40], [100, 70], peaked=peaked, name="float32")
        p.check(*p.run(scale=scale), scale=scale)
    p = Problem(torch, L, np.random.default_rng(3), [3, 40], [100, 70])
    for most in (1, 50, 64, 99, 100, 5000):
        p.check(*p.run(max_len=most), max_len=most)


def test_bad_pages(env):  # noqa: F811
    """Pages whose number is none of the cache's are seen by no row, and a row of only such gives zeros."""
    torch, L = env
    bad = [(0, 1, -1), (0, 4, 10 ** 6), (1, 0, 2 ** 31 - 1), (2, 0, -2 ** 31), (2, 1, 10 ** 8)]
    for group, new in ((2, [3, 1, 2]), (16, [30, 20, 20])):
        p = Problem(torch, L, np.random.default_rng(4), new, [150, 60, 25], bad=bad, group=group)
        p.check(*p.run())


@pytest.mark.parametrize("case", [(1, 9000, 1, 8, 128, "bfloat16"), (3, 20000, 2, 1, 64, "float16"),
                                  (40, 5000, 1, 4, 128, "float32"), (2, 3500, 1, 2, 256, "bfloat16")], ids=str)
def test_split_keys(env, case):  # noqa: F811
    """Long sequences split over workgroups: joined to the oracle's result, the same bits at every call."""
    torch, L = env
    new, length, heads, group, dim, name = case
    rng = np.random.default_rng(length)
    p = Problem(torch, L, rng, [new, 1, 0], [length, 130, 64], heads=heads, group=group, dim=dim, page=64, name=name,
                kind=q8.F32)
    assert L.ds_attn8_work(p.q, p.cache, p.chunk) > 0
    out, lse = p.run()
    some = {(t, h) for t in (0, new - 1, new) for h in (0, heads * group - 1)}
    p.check(out, lse, rows=some)
    for _ in range(3):
        again, sums = p.run()
        assert torch.equal(out, again) and torch.equal(lse, sums)
    work = torch.full((L.ds_attn8_work(p.q, p.cache, p.chunk) + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    again, sums = p.run(work=work)                                   # whatever the workspace held
    assert torch.equal(out, again) and torch.equal(lse, sums)
    p.check(*p.run(window=3000), window=3000, rows=some)
    one, _ = p.run(max_len=length)
    p.check(one, rows=some)


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.E5M2])
@pytest.mark.parametrize("group", [1, 16])
@pytest.mark.parametrize("kind", [q8.POW2, q8.F32])
def test_not_numbers_in_masked_places(env, fmt, group, kind):  # noqa: F811
    """Keys and values of NaN (and of infinity in e5m2) reach the rows that see them and no others."""
    torch, L = env
    new, length = 40, 101
    p = Problem(torch, L, np.random.default_rng(5), [new], [length], fmt=fmt, group=group, dim=48, page=16, kind=kind)
    base = length - new
    infinite = 0x7C if fmt == q8.E5M2 else 0x7F
    marks = [(70, 0, 0x7F), (85, 5, infinite), (85, 6, infinite | 0x80), (90, 5, 0x7F), (3, 1, 0x7F), (95, 7, infinite),
             (96, 7, infinite | 0x80)]
    for j, d, code in marks:
        page, off = attn8.place(p.table[0], j, 16, p.pages)
        p.codes[1][page, :, off, d] = code
    p.put()
    out, lse = p.run(window=30)
    got = out.double().cpu().numpy()
    (k, _), (v, _) = p.values(0, 0, length), p.values(1, 0, length)
    j = np.arange(length)
    for i in range(new):
        pos = base + i
        sees = (j <= pos) & (j > pos - 30)
        seen = v[sees, 0]
        for h in range(2 * group):
            kv = h // group
            want, lim, total, off = p.row(p.eq[i, h], k[:, kv], np.where(np.isfinite(v[:, kv]), v[:, kv], 0.0), sees, 48 ** -0.5)
            assert abs(float(lse[i, h]) - total) <= off
            for d in range(48):
                special = seen[~np.isfinite(seen[:, d]), d]
                if len(special) == 0:
                    assert abs(got[i, h, d] - want[d]) <= lim[d], (i, h, d)
                else:
                    with np.errstate(invalid="ignore"):
                        s = special.sum()
                    assert np.isnan(got[i, h, d]) if np.isnan(s) else got[i, h, d] == s, (i, h, d, s)
    # a key that is no number: its rows are none, the others stay as they are
    page, off = attn8.place(p.table[0], 80, 16, p.pages)
    for j, d, code in marks:
        at = attn8.place(p.table[0], j, 16, p.pages)
        p.codes[1][at[0], :, at[1], d] = 0
    p.codes[0][page, :, off, 2] = 0x7F
    p.put()
    out, lse = p.run()
    for i in range(new):
        assert bool(torch.isnan(out[i]).all()) == (base + i >= 80) and not (base + i < 80 and torch.isnan(out[i]).any())
        assert bool(torch.isnan(lse[i]).all()) == (base + i >= 80)


def test_strides(env):  # noqa: F811
    """Queries inside one projection's rows, unaligned ones, outputs in heads' order."""
    torch, L = env
    for lists in (([2, 5], [70, 40]), ([150], [150])):
        p = Problem(torch, L, np.random.default_rng(6), *lists, heads=2, group=3, dim=80)
        want, sums = p.run()
        wide = torch.randn(p.tokens, 11, 84, device="cuda").to(p.q.dtype)
        for d in (0, 3):
            wide[:, 2:8, d:d + 80] = p.q
            q = wide[:, 2:8, d:d + 80]
            out = torch.full((6, p.tokens, 80), 5.0, dtype=q.dtype, device="cuda").transpose(0, 1)
            L.ds_attn8(q, p.cache, p.chunk, out)
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            into = wide.clone()
            L.ds_attn8(q, p.cache, p.chunk, into[:, 2:8, d:d + 80])
            torch.cuda.synchronize()
            mine = (p.starts[0], p.starts[-1])
            assert torch.equal(into[mine[0]:mine[1], 2:8, d:d + 80], want[mine[0]:mine[1]])
            into[mine[0]:mine[1], 2:8, d:d + 80] = wide[mine[0]:mine[1], 2:8, d:d + 80]
            assert torch.equal(into, wide)


def test_other_streams_and_threads(env):  # noqa: F811
    """Two calls at once on streams of their own, with workspaces of their own."""
    torch, L = env
    ps = [Problem(torch, L, np.random.default_rng(s), [1, 2], [4000 + s, 3000], group=4, page=64) for s in (1, 2)]
    want = [p.run() for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    outs = [[torch.zeros_like(w) for w in ws] for ws in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for p, st, o in zip(ps, streams, outs):
            L.ds_attn8(p.q, p.cache, p.chunk, *o, stream=st)
        for p, st, o in zip(ps, streams, outs):
            L.ds_attn8(p.q, p.cache, p.chunk, *o, stream=int(st.cuda_stream))
    torch.cuda.synchronize()
    for p, o, w in zip(ps, outs, want):
        rows = slice(0, int(p.starts[-1]))
        assert torch.equal(o[0][rows], w[0][rows]) and torch.equal(o[1][rows], w[1][rows])


def test_captured(env):  # noqa: F811
    """A graph of a whole step follows its lists from replay to replay, beside another graph."""
    torch, L = env
    rng = np.random.default_rng(12)
    graphs = []
    for seed in (0, 1):
        p = Problem(torch, L, np.random.default_rng(seed), [1, 1, 1], [2500, 70, 15], group=4, dim=64, page=16, cols=200,
                    extra=400, behind=0, name="float32")
        kv = [torch.from_numpy(rng.standard_normal((3, 2, 64)).astype(np.float32)).cuda() for _ in range(2)]
        turned = [torch.empty_like(p.q), torch.empty_like(kv[0])]
        pos = (p.lists[1] - 1).contiguous()
        freqs = torch.from_numpy((1e4 ** (-np.arange(32) / 32)).astype(np.float32)).cuda()
        out, lse = torch.empty_like(p.q), torch.empty(3, 8, device="cuda")

        def step(p=p, kv=kv, turned=turned, pos=pos, freqs=freqs, out=out, lse=lse):
            L.ds_rotary(p.q, pos, freqs, turned[0])
            L.ds_rotary(kv[0], pos, freqs, turned[1])
            L.ds_cache8_write(p.cache, p.chunk, turned[1], kv[1])
            L.ds_attn8(turned[0], p.cache, p.chunk, out, lse)
        g = torch.cuda.CUDAGraph()
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            step()
        graphs.append((g, p, kv, pos, out, lse, step))
    for i in range(4):
        for g, p, kv, pos, out, lse, step in graphs:
            # a token more, in pages of its own
            p.lists[1].add_(1)
            pos.add_(1)
            n = p.lists[1].cpu().numpy()
            for b in range(3):
                if (n[b] - 1) % 16 == 0:
                    p.lists[2][b, (n[b] - 1) // 16] = p.pages - 1 - 3 * i - b
            p.q.normal_()
            for x in kv:
                x.normal_()
            out.fill_(float("nan"))
            lse.fill_(float("nan"))
        torch.cuda.synchronize()
        for g, *_ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, p, kv, pos, out, lse, step in graphs:
            a, b = out.clone(), lse.clone()
            out.fill_(float("nan"))
            step()                                                  # eager, on the same lists
            torch.cuda.synchronize()
            assert torch.equal(a, out) and torch.equal(b, lse) and not torch.isnan(a).any(), i


def test_run_of_a_prompt_and_tokens(env):  # noqa: F811
    """Prompts in chunks, then tokens one by one, through positions, cache and attention: the oracle's whole
    attention over the values that the cache then holds."""
    torch, L = env
    rng = np.random.default_rng(13)
    heads, group, dim, page, seqs = 2, 3, 64, 16, 3
    cache = L.Cache8(40, heads, dim, page)
    table = torch.from_numpy(rng.permutation(40)[:30].reshape(seqs, 10).astype(np.int32)).cuda()
    freqs = (1e4 ** (-np.arange(32) / 32)).astype(np.float32)
    f = torch.from_numpy(freqs).cuda()
    length = np.zeros(seqs, np.int64)
    keys = [[] for _ in range(seqs)]
    steps = [[50, 3, 20], [30, 0, 45], [0, 9, 1]] + [[1, 1, 1]] * 4
    for new in steps:
        starts = np.concatenate([[0], np.cumsum(new)])
        length += new
        tokens = int(starts[-1])
        pos = np.concatenate([np.arange(n - m, n) for n, m in zip(length, new)]).astype(np.int32)
        qkv, exact = typed(torch, rng.standard_normal((tokens, heads * (group + 2), dim)), "bfloat16")
        q, k, v = qkv.split([heads * group, heads, heads], 1)
        chunk = L.Chunk(*(torch.from_numpy(np.asarray(a, np.int32)).cuda() for a in (starts, length)), table)
        both = qkv[:, :heads * (group + 1)]
        L.ds_rotary(both, torch.from_numpy(pos).cuda(), f)
        L.ds_cache8_write(cache, chunk, k, v)
        out = torch.empty_like(q)
        L.ds_attn8(q, cache, chunk, out)
        torch.cuda.synchronize()
        ek, ev = (x.double().cpu().numpy() for x in cache.values())
        want = attn8.rotary(exact[:, :heads * (group + 1)], pos, freqs)
        turned = both.double().cpu().numpy()
        assert (np.abs(turned - want) <= np.abs(want) * HALF["bfloat16"] + 2.0 ** -18 * np.abs(exact).max()).all()
        t = table.cpu().numpy()
        for b in range(seqs):
            j = np.arange(length[b])
            kb, vb = (x[t[b, j // page], :, j % page] for x in (ek, ev))
            for i in range(starts[b], starts[b + 1]):
                for h in range(heads * group):
                    row, _, room, p = attn8.attend(turned[i, h], kb[:, h // group], vb[:, h // group], j <= pos[i], dim ** -0.5)
                    # as above, with 2^-12 over all of fp32's roundings (300 keys of 64 values)
                    lim = room * (WEIGHT["bfloat16"] + 2.0 ** -12) + np.abs(row) * HALF["bfloat16"]
                    assert (np.abs(out[i, h].double().cpu().numpy() - row) <= lim * 1.01).all()
                    # what was written is the turned key, to half a step of e4m3 (2^-4) and the scale's slack
                    if h % group == 0:
                        kk = turned[i, heads * group + h // group]
                        assert (np.abs(kb[pos[i], h // group] - kk) <= np.abs(kk) * 2.0 ** -4 + np.abs(kk).max() * 2.0 ** -9).all()
