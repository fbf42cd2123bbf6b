"""The paged cache (FMACache: append, attend, step) against a plain float64
evaluation of causal FMA over whole sequences (cache_reference.py, which
derives the bounds), in ragged batches of pieces and single tokens."""
import random

import pytest
import torch

import cache_reference as R
import oracle
import paper_2310_11960_amd as F

pytestmark = pytest.mark.gpu


def _dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


class Served:
    """Sequences of known tokens that enter a cache piece by piece."""

    def __init__(self, lens, heads=4, kv_heads=2, d=64, r=64, rank=1, max_len=None, dtype=torch.bfloat16, seed=1,
                 scale=0.0, shared=False, spare=3, amp=1.0):
        self.dev = _dev()
        self.lens, self.r, self.rank, self.dtype, self.scale = lens, r, rank, dtype, scale
        self.H, self.kv, self.d = heads, kv_heads, d
        self.max_len = max_len or max(max(lens), 1)
        self.op = F.FMACache(heads, self.max_len, kv_heads=kv_heads, head_dim=d, block=r, dtype=dtype, rank=rank,
                             weights_per_head=not shared, softmax_scale=scale)
        self.levels = R.levels_of(self.max_len, r)
        assert self.op.sets == self.levels * rank and self.op.weights_len == R.weight_len(self.max_len, r, rank)
        g = torch.Generator().manual_seed(seed)
        mk = lambda h, n: (amp * torch.randn(n, h, d, generator=g)).to(dtype)  # noqa: E731
        self.q, self.k, self.v = ([mk(h, n) for n in lens] for h in (heads, kv_heads, kv_heads))
        sc = torch.cat([torch.full((rank * (r << l),), (r << l) ** -0.5) for l in range(self.levels)] or [torch.empty(0)])
        shape = (self.op.weights_len,) if shared else (kv_heads, self.op.weights_len)
        self.wk, self.wv = (torch.randn(shape, generator=g) * sc for _ in range(2))
        blocks = max(self.op.blocks, 1)
        need = sum(-(-n // r) for n in lens)
        order = list(range(need + spare))
        random.Random(seed).shuffle(order)
        self.table = torch.full((len(lens), blocks), -1, dtype=torch.int32)
        at = 0
        for i, n in enumerate(lens):
            for b in range(-(-n // r)):
                self.table[i, b] = order[at]
                at += 1
        self.stable = torch.where(self.table >= 0, (self.table + 7) % (need + spare), self.table)
        self.pages = self.op.new_pages(need + spare, need + spare, self.dev)
        for t in self.pages:
            if t is not None:
                t.fill_(float("nan"))          # nothing that was not written may be read
        self.have = [0] * len(lens)

    def batch(self, take, start=None, max_chunk=None, table=None, stable=None):
        cu = torch.tensor([0] + take, dtype=torch.int32).cumsum(0).to(torch.int32)
        put = lambda t: t.to(self.dev)  # noqa: E731
        return F.CacheBatch(put(cu), put(torch.tensor(self.have if start is None else start, dtype=torch.int32)),
                            put(self.table if table is None else table), put(self.stable if stable is None else stable),
                            max(take) if max_chunk is None else max_chunk)

    def rows(self, x, take, start=None, pad=0):
        start = self.have if start is None else start
        t = [y[s:s + n] for y, s, n in zip(x, start, take)] + [torch.full((pad,) + x[0].shape[1:], float("nan"), dtype=self.dtype)]
        return torch.cat(t).to(self.dev)

    def weights(self):
        return self.wk.to(self.dev), self.wv.to(self.dev)

    def step(self, take, how="step", pad=0, **kw):
        b = self.batch(take, **kw)
        q, k, v = (self.rows(x, take, pad=pad) for x in (self.q, self.k, self.v))
        out = torch.full_like(q, 7.0)
        if how == "step":
            self.op.step(q, k, v, *self.weights(), self.pages, b, out=out)
        else:
            self.op.append(k, v, *self.weights(), self.pages, b)
            if how == "two":
                self.op.attend(q, self.pages, b, out=out)
        if how != "append":
            self.check(out, take)
            assert (out[sum(take):] == 7.0).all()
        self.have = [h + t for h, t in zip(self.have, take)]

    def reference(self, i, h, lo, hi):
        g = self.H // self.kv
        w = (self.wk, self.wv) if self.wk.dim() == 1 else (self.wk[h // g], self.wv[h // g])
        return R.attend(self.q[i][lo:hi, h], self.k[i][:hi, h // g], self.v[i][:hi, h // g], *w, self.r, self.rank,
                        self.levels, self.scale or self.d ** -0.5, self.dtype, lo=lo)

    def check(self, out, take):
        got, at = out.double().cpu(), 0
        for i, (s, t) in enumerate(zip(self.have, take)):
            for h in sorted({0, self.H // 2, self.H - 1}) if t else []:
                ref, bound = self.reference(i, h, s, s + t)
                bad = ((got[at:at + t, h] - ref).abs() - bound).max()
                assert bad <= 0, "sequence %d head %d at %d + %d: over the bound by %.3g" % (i, h, s, t, float(bad))
            at += t

    def check_pages(self):
        """Every written row and every complete block's sums."""
        kp, vp = self.pages.k.cpu(), self.pages.v.cpu()
        for i, n in enumerate(self.have):
            for b in range(-(-n // self.r)):
                p, c = int(self.table[i, b]), min(self.r, n - b * self.r)
                for pool, src in ((kp, self.k), (vp, self.v)):
                    assert torch.equal(pool[p][:, :c].transpose(0, 1), src[i][b * self.r:b * self.r + c])
            if not self.op.sets:
                continue
            sums = self.pages.summaries.cpu().double()
            for h in range(self.kv):
                for x, (src, w) in enumerate(((self.k, self.wk), (self.v, self.wv))):
                    ref, mag = R.running_sums(src[i][:n, h], w if w.dim() == 1 else w[h], self.r, self.rank, self.levels)
                    for b in range(n // self.r):
                        got = sums[int(self.stable[i, b]), h, x]
                        bound = (self.r + (1 << max(self.levels - 1, 0)) + 8) * R.U * mag[b]
                        assert ((got - ref[b]).abs() <= bound).all(), (i, h, x, b)


DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SHAPES = [  # heads, kv_heads, d, r, rank
    (4, 2, 64, 64, 1), (3, 3, 32, 16, 2), (8, 1, 128, 128, 1), (6, 2, 64, 192, 1), (2, 2, 128, 32, 4), (40, 1, 32, 64, 1),
    (2, 1, 64, 256, 2),
]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("how", ["step", "two"])
def test_pieces_and_tokens(shape, dtype, how):
    H, kv, d, r, rank = shape
    s = Served([9 * r + 5, 3 * r, 1, 6 * r + 1], H, kv, d, r, rank, dtype=DT[dtype])
    s.step([3, 0, 1, r], how)                       # first tokens, an absent sequence, a whole block
    s.step([r - 3, 1, 0, 1], how, pad=2)            # a block completed, rows behind the last sequence
    s.step([1, r - 1, 0, 2], how)                   # first token of a block; a block completed by a piece
    s.step([3 * r + 7, 2 * r, 0, r], how)           # pieces over several blocks
    s.step([1, 0, 0, 3 * r - 2], how, pad=1)
    s.step([r, 0, 0, 0], how)
    s.step([4 * r - 4, 0, 0, r], how)
    assert s.have == [9 * r + 5, 3 * r, 1, 6 * r + 1]
    s.check_pages()


ROWS = [  # as above, with key heads enough that the device's waves take rows
    (32, 32, 64, 64, 1), (32, 16, 32, 16, 2), (48, 16, 128, 128, 1), (40, 8, 64, 192, 1), (64, 64, 128, 32, 4),
    (66, 2, 32, 64, 1), (32, 16, 64, 256, 2),
]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", ROWS, ids=lambda s: "-".join(map(str, s)))
def test_longer_pieces(shape, dtype):
    """Pieces of enough rows that the waves of a workgroup take different ones."""
    H, kv, d, r, rank = shape
    n = max(9 * r + 5, 1200)
    s = Served([n, n // 2, 40, 1], H, kv, d, r, rank, dtype=DT[dtype])
    s.step([n - r - 3, n // 2 - 50, 40, 0], pad=3)
    s.step([r, 33, 0, 1], "two")
    s.step([3, 17, 0, 0])
    s.check_pages()


@pytest.mark.parametrize("dtype", list(DT))
def test_longer_pieces_with_missing_pages(dtype):
    """A missing page hides its tokens there too; rows of no sequence stay."""
    r, n, kv = 32, 900, 16
    s = Served([n], kv, kv, 64, r, 1, dtype=DT[dtype])
    s.step([n], "append")
    q, b = s.rows(s.q, [n], start=[0], pad=2), s.batch([n], start=[0])
    gone = (3, 4, 11)
    for x in gone:
        b.page_table[0, x] = -1 if x != 4 else s.pages.k.shape[0]
    out = torch.full_like(q, 7.0)
    s.op.attend(q, s.pages, b, out=out)
    assert (out[n:] == 7.0).all()
    for h in (0, kv - 1):
        ref, bound = R.attend(s.q[0][:, h], s.k[0][:, h], s.v[0][:, h], s.wk[h], s.wv[h], r, 1, s.levels, 64 ** -0.5,
                              DT[dtype], missing=gone)
        assert ((out[:n, h].double().cpu() - ref).abs() <= bound).all()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("pieces", [(37, 100, 3), (70, 300, 1), (129, 128, 60), (1, 64, 200), (380, 1, 2)],
                         ids=lambda p: "-".join(map(str, p)))
def test_sums_over_many_blocks(pieces, dtype):
    """Groups of 128 and 256 blocks whose sums cross several calls, at and away
    from the multiples of 64 blocks where the walk over them is cut."""
    r = 16
    lens = [r * p + x for p, x in zip(pieces, (5, 0, -2))]
    s = Served([sum(lens), r * 40 + 3], 2, 1, 32, r, 1, max_len=r * 512, dtype=DT[dtype], seed=14)
    s.step([lens[0], 0], "append")
    s.step([lens[1], r * 40], "append")
    s.step([lens[2], 3])
    s.check_pages()


@pytest.mark.parametrize("dtype", list(DT))
def test_token_by_token(dtype):
    s = Served([16 * 11 + 3, 16 * 4], 2, 1, 32, 16, 1, max_len=16 * 16, dtype=DT[dtype], seed=2)
    s.step([16 * 3 - 2, 0], "append")
    for i in range(16 * 8 + 5):
        s.step([1, 1 if i < 64 else 0])
    s.check_pages()


@pytest.mark.parametrize("dtype", list(DT))
def test_shared_weights_scales_and_lengths_without_levels(dtype):
    s = Served([150, 90], 4, 4, 64, 64, 2, max_len=500, dtype=DT[dtype], scale=-0.2, shared=True)
    s.step([140, 64])
    s.step([10, 26])
    s.check_pages()
    s = Served([100, 3], 2, 2, 64, 64, 1, max_len=128, dtype=DT[dtype])   # two blocks: no coarse level
    assert s.op.sets == 0
    s.step([63, 1])
    s.step([1, 1])
    s.step([36, 1], "two")
    s.check_pages()


def test_large_scores():
    """Scores of several hundreds: the running maxima keep the weights finite."""
    s = Served([64 * 6], 2, 2, 64, 64, 1, dtype=torch.float32, amp=6.0)
    s.step([64 * 4 + 9])
    s.step([1])
    s.step([64])


@pytest.mark.parametrize("dtype,rank", [("bf16", 1), ("f32", 4)])
def test_whole_prompt_equals_the_dense_forward(dtype, rank):
    """One prompt at once, in pieces and by the dense causal pass; and the oracle."""
    r, nb, H = 64, 12, 3
    s = Served([r * nb], H, H, 64, r, rank, dtype=DT[dtype], seed=4)
    att = F.FMA(ndim=1, batch=1, heads=H, seq_len=r * nb, block=r, causal=True, dtype=DT[dtype], rank=rank)
    lay = lambda x: x[0].transpose(0, 1)[None].contiguous().to(s.dev)  # noqa: E731
    dense = att.forward(lay(s.q), lay(s.k), lay(s.v), *s.weights())[0].transpose(0, 1)
    b = s.batch([r * nb])
    out = s.op.step(*(s.rows(x, [r * nb]) for x in (s.q, s.k, s.v)), *s.weights(), s.pages, b)
    tol = 1e-5 if dtype == "f32" else 2e-2
    for h in range(H):
        f = lambda x: x[0][:, h].double().numpy()  # noqa: E731
        ref = oracle.forward_1d(f(s.q), f(s.k), f(s.v), r, s.wk[h].double().numpy(), s.wv[h].double().numpy(),
                                causal=True, rank=rank)
        ref = torch.from_numpy(ref)
        for x in (out, dense):
            assert (x[:, h].double().cpu() - ref).abs().max() <= tol * ref.abs().max()
    # a prompt that entered from the dense layout answers alike
    s2 = Served([r * nb], H, H, 64, r, rank, dtype=DT[dtype], seed=4)
    cut = r * (nb - 2) + 11
    s2.op.append(lay(s.k)[0].transpose(0, 1)[:cut], lay(s.v)[0].transpose(0, 1)[:cut], *s.weights(), s2.pages, s2.batch([cut]))
    s2.have = [cut]
    s2.step([1])
    s2.step([r - 12])


@pytest.mark.parametrize("dtype", list(DT))
def test_pages_behind_are_not_read(dtype):
    """Token pages before the previous block and sums that no later query
    reads may be freed (and overwritten)."""
    r, n = 32, 32 * 21 + 9
    s = Served([n], 2, 1, 64, r, 1, max_len=32 * 32, dtype=DT[dtype])
    s.step([n - 40], "append")
    for take in (1, 5, 34):
        b0, b1 = s.have[0] // r, (s.have[0] + take - 1) // r
        keep = set(range(max(0, b0 - 1), b1 + 1))
        skeep = keep | {x for b in range(b0, b1 + 1) for x, _ in R.far_rows(b, s.levels, 1)}
        table, stable = s.table.clone(), s.stable.clone()
        for b in range(table.shape[1]):
            if b not in keep and table[0, b] >= 0:
                s.pages.k[int(table[0, b])] = float("nan")
                table[0, b] = -1 if b % 2 else 1 << 30
            if b not in skeep and stable[0, b] >= 0:
                s.pages.summaries[int(stable[0, b])] = float("nan")
                stable[0, b] = -5
        s.step([take], table=table, stable=stable)


@pytest.mark.parametrize("dtype", list(DT))
def test_missing_pages_hide_their_tokens(dtype):
    r = 32
    s = Served([r * 2 + 7], 2, 2, 64, r, 1, max_len=64 * 8, dtype=DT[dtype])
    s.step([r * 2 + 4], "append")
    q = s.rows(s.q, [3])
    ref = lambda gone, h: R.attend(s.q[0][68:71, h], s.k[0][:71, h], s.v[0][:71, h], s.wk[h], s.wv[h], r, 1, s.levels,  # noqa: E731
                                   64 ** -0.5, DT[dtype], lo=68, missing=gone)
    k, v = s.rows(s.k, [3]), s.rows(s.v, [3])
    s.op.append(k, v, *s.weights(), s.pages, s.batch([3]))
    for gone in ((1,), (2,), (1, 2)):
        table = s.table.clone()
        for b in gone:
            table[0, b] = -1
        out = s.op.attend(q, s.pages, s.batch([3], table=table)).double().cpu()
        for h in range(2):
            want, bound = ref(gone, h)
            assert ((out[:, h] - want).abs() <= bound).all()
    gone = torch.full_like(s.table, -1)
    assert not s.op.attend(q, s.pages, s.batch([3], table=gone, stable=gone)).any()     # rows that see nothing
    # a call's own tokens are seen wherever their page is, and not kept
    before = s.pages.k.clone()
    table = torch.full_like(s.table, -1)
    out = s.op.step(q, k, v, *s.weights(), s.pages, s.batch([3], table=table, stable=table)).double().cpu()
    assert torch.equal(before.nan_to_num(9.0), s.pages.k.nan_to_num(9.0))
    one = v[0].double().cpu()
    assert ((out[0] - one).abs() <= 2 * R.HALF[DT[dtype]] * one.abs()).all()      # the first sees itself alone


ODD = [(2, 2, 64, 64, [100, 3], [4, 3]), (4, 2, 32, 16, [20, 40], [13, 16]), (4, 2, 64, 64, [70, 0], [5, 60]),
       (8, 2, 128, 64, [64, 130], [40, 62]), (16, 16, 64, 64, [30, 64] * 4, [300, 128] * 4),
       (16, 16, 32, 16, [7, 64] * 4, [190, 128] * 4), (8, 4, 128, 128, [130, 64] * 4, [300, 128] * 4)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", ODD, ids=lambda s: "-".join(map(str, s[:4] + (len(s[4]),))))
@pytest.mark.parametrize("what", ["values", "keys"])
def test_no_number_reaches_an_earlier_query(shape, dtype, what):
    # an infinity and a NaN among a piece's own tokens: in a value's channel they stay in
    # that channel of the queries from the token on; in a key, in those queries
    heads, kv, d, r, before, take = shape
    s = Served([a + b for a, b in zip(before, take)], heads, kv, d, r, max_len=1000, dtype=DT[dtype], seed=43)
    s.step(before) if any(before) else None
    at = [(n // 3, n - n // 4 - 1) for n in take]     # (row of the piece, its odd tokens)
    q, k, v = (s.rows(x, take) for x in (s.q, s.k, s.v))
    off = [sum(take[:i]) for i in range(len(take))]
    for o, (j0, j1) in zip(off, at):
        if what == "values":
            v[o + j0, :, 5], v[o + j1, :, d - 3] = float("inf"), float("nan")
        else:
            k[o + j0, :, 5], k[o + j1, :, d - 3] = float("nan"), float("inf")
    out = torch.full_like(q, 7.0)
    s.op.step(q, k, v, *s.weights(), s.pages, s.batch(take), out=out)
    out = out.cpu().double()
    for i, (o, (j0, j1), n) in enumerate(zip(off, at, take)):
        for h in range(0, heads, max(1, heads // 4)):
            ref, bound = s.reference(i, h, before[i], before[i] + n)
            got, good = out[o:o + n, h], torch.ones(n, d, dtype=torch.bool)
            if what == "values":
                good[j0:, 5] = False
                good[j1:, d - 3] = False
                assert not torch.isfinite(got[~good]).any(), (i, h)
            else:
                good[j0:] = False
                assert torch.isnan(got[j0:]).all(), (i, h)
            bad = ((got - ref).abs() > bound) | ~torch.isfinite(got)
            assert not (bad & good).any(), (i, h, (bad & good).nonzero()[:4].tolist())


def test_sequences_that_do_not_fit_are_skipped():
    r = 32
    s = Served([100, 100, 100, 100, 100, 100], 2, 2, 64, r, 1, max_len=128)
    q, k, v = (torch.cat([x[i][:20] for i in range(6)]).to(s.dev) for x in (s.q, s.k, s.v))
    cu = torch.tensor([0, 20, 40, 60, 80, 100, 130], dtype=torch.int32, device=s.dev)      # the last: past the rows
    start = torch.tensor([0, -1, 109, 0, 0, 0], dtype=torch.int32, device=s.dev)           # negative, past max_len
    b = F.CacheBatch(cu, start, s.table.to(s.dev), s.stable.to(s.dev), 20)
    out = torch.full_like(q, 3.0)
    s.op.step(q, k, v, *s.weights(), s.pages, b, out=out)
    for i, fine in enumerate((True, False, False, True, True, False)):
        rows = out[20 * i:20 * (i + 1)]
        assert (rows != 3.0).any() if fine else (rows == 3.0).all(), i
        page = s.pages.k[int(s.table[i, 0])]
        assert torch.isfinite(page[:, :20]).all() if fine else torch.isnan(page).all(), i
    before = out.clone()
    for chunk, bad in ((19, cu), (20, torch.flip(cu, [0]))):                               # longer than named; falling
        s.op.step(q, k, v, *s.weights(), s.pages, b._replace(max_chunk=chunk, cu_tokens=bad), out=out)
        s.op.append(k, v, *s.weights(), s.pages, b._replace(max_chunk=chunk, cu_tokens=bad))
        assert torch.equal(out, before)
    # a table too narrow for the length
    narrow = b._replace(start=torch.full_like(start, 13), page_table=s.table[:, :1].contiguous().to(s.dev),
                        summary_table=s.stable[:, :1].contiguous().to(s.dev))
    s.op.step(q, k, v, *s.weights(), s.pages, narrow, out=out)
    assert torch.equal(out, before)


@pytest.mark.parametrize("dtype", list(DT))
def test_ragged_batches_of_many_sequences(dtype):
    """One long piece among many short ones: workgroups that search their tile."""
    r = 16
    lens = [1 + (7 * i) % 5 for i in range(150)]
    lens[77], lens[3] = 700, 0
    s = Served(lens, 2, 1, 32, r, 1, max_len=1024, dtype=DT[dtype], seed=6)
    s.step([max(0, n - 1) for n in lens])
    s.step([min(1, n) for n in lens])
    s.check_pages()


def test_repeats_and_going_back():
    r = 32
    s = Served([r * 7], 4, 2, 64, r, 2, seed=7)
    s.step([r * 4 + 3])
    args = lambda n: [s.rows(x, [n]) for x in (s.q, s.k, s.v)]  # noqa: E731
    first = s.op.step(*args(2 * r + 1), *s.weights(), s.pages, s.batch([2 * r + 1]))
    sums = s.pages.summaries.clone()
    # other tokens in their place, then the same ones again
    g = torch.Generator().manual_seed(1)
    junk = [torch.randn(x.shape, generator=g).to(x) for x in args(2 * r + 1)]
    s.op.step(*junk, *s.weights(), s.pages, s.batch([2 * r + 1]))
    for _ in range(2):
        again = s.op.step(*args(2 * r + 1), *s.weights(), s.pages, s.batch([2 * r + 1]))
        assert torch.equal(first, again)
        assert torch.equal(sums.nan_to_num(5.0), s.pages.summaries.nan_to_num(5.0))


def test_shared_prompt_pages():
    """Two continuations of one prompt, its pages and sums held once."""
    r = 32
    s = Served([r * 5 + 9, r * 5 + 9], 2, 2, 64, r, 1, seed=8)
    for x in (s.q, s.k, s.v):
        x[1][:r * 4] = x[0][:r * 4]
    s.table[1, :4], s.stable[1, :4] = s.table[0, :4], s.stable[0, :4]
    s.step([r * 4, 0], "append")
    s.have = [r * 4, r * 4]
    s.step([r, 3])
    s.step([9, r + 6])


@pytest.mark.parametrize("dtype", list(DT))
def test_strided_rows_and_streams(dtype):
    """Heads of one packed projection in, a padded output, another stream."""
    r = 64
    s = Served([200, 70], 4, 2, 64, r, 1, max_len=512, dtype=DT[dtype], seed=9)
    s.step([130, 60], "append")
    take = [70, 10]
    want = s.op.step(*(s.rows(x, take) for x in (s.q, s.k, s.v)), *s.weights(), s.pages, s.batch(take))
    packed = torch.cat([s.rows(x, take) for x in (s.q, s.k, s.v)], 1)
    wide = torch.full((80, 9, 64), 5.0, dtype=DT[dtype], device=s.dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b, w = s.batch(take), s.weights()
    torch.cuda.synchronize()
    s.op.step(packed[:, :4], packed[:, 4:6], packed[:, 6:], *w, s.pages, b, out=wide[:, 1:8:2], stream=side)
    side.synchronize()
    assert torch.equal(wide[:, 1:8:2], want)
    assert (wide[:, 0::2] == 5.0).all()
    q = s.rows(s.q, take)                                                   # in place of the queries
    s.op.attend(q, s.pages, b, out=q)
    s.check(q, take)


def test_graph_replays_with_other_lengths():
    r = 32
    s = Served([r * 9, r * 9, r * 9], 4, 2, 64, r, 1, seed=10)
    s.step([r * 5, 17, 1], "append")
    for shapes in ([(1, 1, 1), (1, 0, 1), (0, 1, 1)], [(70, 3, 0), (1, 66, 1), (20, 20, 33)]):
        most, rows = max(map(max, shapes)), 80
        buf = [torch.zeros(rows, h, 64, dtype=s.dtype, device=s.dev) for h in (4, 2, 2)]
        out = torch.zeros_like(buf[0])
        first = s.batch(list(shapes[0]), max_chunk=most)
        b = F.CacheBatch(*[t.clone() for t in first[:4]], most)
        w = s.weights()
        s.op.step(*buf, *w, s.pages, b._replace(cu_tokens=torch.zeros_like(b.cu_tokens)), out=out)   # warm, nothing new
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.op.step(*buf, *w, s.pages, b, out=out)
        for take in shapes:
            take = list(take)
            for t, x in zip(buf, (s.q, s.k, s.v)):
                t.zero_()
                new = s.rows(x, take)
                t[:new.shape[0]] = new
            now = s.batch(take, max_chunk=most)
            for t, x in zip(b[:4], now[:4]):
                t.copy_(x)
            out.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            s.check(got, take)
            assert (got[sum(take):] == 7.0).all()
            eager = s.op.step(*buf, *w, s.pages, b)
            assert torch.equal(eager[:sum(take)], got[:sum(take)])
            s.have = [h + t for h, t in zip(s.have, take)]


@pytest.mark.parametrize("dtype", list(DT))
def test_graph_replays_of_longer_pieces(dtype):
    r, H, rows, most = 64, 16, 2300, 1200
    s = Served([r * 40, r * 40], H, H, 128, r, 2, dtype=DT[dtype], seed=44)
    s.step([100, 700], "append")
    w = s.weights()
    buf = [torch.zeros(rows, H, 128, dtype=s.dtype, device=s.dev) for _ in range(3)]
    out = torch.zeros_like(buf[0])
    b = s.batch([0, 0], max_chunk=most)
    s.op.step(*buf, *w, s.pages, b, out=out)   # warm, nothing new
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.op.step(*buf, *w, s.pages, b, out=out)
    for take in ([1100, 1100], [1200, 1], [0, 600]):
        for t, x in zip(buf, (s.q, s.k, s.v)):
            new = s.rows(x, take)
            t[:new.shape[0]] = new
        for t, x in zip(b[:4], s.batch(take, max_chunk=most)[:4]):
            t.copy_(x)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        s.check(got, take)
        assert (got[sum(take):] == 7.0).all()
        assert torch.equal(s.op.step(*buf, *w, s.pages, b)[:sum(take)], got[:sum(take)])
        s.have = [h + t for h, t in zip(s.have, take)]
    s.check_pages()


def test_pools_past_32_bit_offsets():
    """Pages whose elements lie beyond 2^31 and 2^32 bytes."""
    dev = _dev()
    r, kv, d = 128, 8, 128
    page = kv * r * d                                 # 2^17 elements
    n = 2 ** 31 // page + 5
    s = Served([r * 3 + 20], 8, kv, d, r, 1, seed=11)
    s.pages = F.CachePages(torch.empty(n, kv, r, d, dtype=s.dtype, device=dev),
                           torch.empty(n, kv, r, d, dtype=s.dtype, device=dev), s.pages.summaries)
    s.table[0, :4] = torch.tensor([n - 1, 3, n - 2, n - 4], dtype=torch.int32)
    s.step([r * 2 + 9])
    s.step([1])
    s.step([r - 1])
    s.check_pages()


def test_prompt_through_norm_rotation_and_cache():
    """What a server runs: a projection's rows normed, rotated and given to the
    cache, piece by piece, against the training path on the whole prompt."""
    dev = _dev()
    r, nb, H, kv, d = 64, 8, 4, 2, 64
    n = r * nb
    g = torch.Generator().manual_seed(12)
    qkv = torch.randn(1, n, H + 2 * kv, d, generator=g).to(dev)
    gq, gk = (1 + 0.2 * torch.randn(d, generator=g).to(dev) for _ in range(2))
    split = lambda x: (x[:, :, :H], x[:, :, H:H + kv], x[:, :, H + kv:])  # noqa: E731
    train = F.QKNormRope(heads=H, kv_heads=kv, dtype=torch.float32, repeat_kv=True)
    att = F.FMA(ndim=1, batch=1, heads=H, seq_len=n, block=r, causal=True, dtype=torch.float32)
    cache = F.FMACache(H, n, kv_heads=kv, block=r, dtype=torch.float32)
    wk, wv = (torch.randn(kv, cache.weights_len, generator=g).to(dev) / 8 for _ in range(2))
    rep = lambda w: w.repeat_interleave(H // kv, 0).contiguous()  # noqa: E731
    want = att.forward(*train.forward(*split(qkv), gq, gk), rep(wk), rep(wv))[0].transpose(0, 1)
    serve = F.QKNormRope(heads=H, kv_heads=kv, dtype=torch.float32)
    pages = cache.new_pages(nb, nb, dev)
    table = torch.randperm(nb, generator=g).to(torch.int32)[None].to(dev)
    at = 0
    for take in (r * 3 + 5, 1, 1, r, r * 2 - 7, n - r * 6):
        rows = qkv[:, at:at + take]
        pos = torch.arange(at, at + take, dtype=torch.int32, device=dev)[None]
        new = [torch.empty(1, take, h, d, device=dev) for h in (H, kv, kv)]
        serve.forward(*split(rows), gq, gk, positions=pos, **{"qkv"[i] + "_out": t.transpose(1, 2) for i, t in enumerate(new)})
        b = F.CacheBatch(torch.tensor([0, take], dtype=torch.int32, device=dev),
                         torch.tensor([at], dtype=torch.int32, device=dev), table, table, take)
        out = cache.step(*(t[0] for t in new), wk, wv, pages, b)
        # two fp32 evaluations, each within 1e-5 of the largest entry
        assert (out - want[at:at + take]).abs().max() <= 2e-5 * want.abs().max()
        at += take
    assert at == n
