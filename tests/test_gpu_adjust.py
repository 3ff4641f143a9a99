"""ppd_adjust_logits against 64 bits, row by row."""
import math
import random

import numpy as np
import pytest
import torch

from paged_common import HALF_STEP, TINY
from paper_2307_05908_amd import binding

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
RULES = ("ids", "history", "history_len", "prompt_len", "repetition", "presence", "frequency", "bias_start", "bias_ids", "bias", "mask", "mask_row")


class Case:
    def __init__(self, rows, vocab, dtype, before=20, biases=0, masks=0, seed=0, pad=0, start=0, stride=0, without=()):
        g, rng = torch.Generator().manual_seed(seed), random.Random(seed)
        self.rows, self.vocab, self.dtype = rows, vocab, dtype
        self.n, seqs = start + sum(rows) + pad, len(rows)
        self.logits = (3 * torch.randn(self.n, max(stride, vocab), generator=g)).to(dtype)[:, :vocab]
        self.row_start = torch.tensor(np.concatenate([[start], start + np.cumsum(rows)]), dtype=torch.int32)

        def words(*shape):
            return torch.randint(-1, min(vocab, 40) + 1, shape, generator=g, dtype=torch.int32) * rng.choice([1, 1, max(1, vocab // 40)])

        self.ids, self.history = words(self.n), words(seqs, before + 3)
        self.history_len = torch.tensor([rng.randint(0, before) for _ in rows], dtype=torch.int32)
        self.prompt_len = torch.tensor([rng.randint(-1, before) for _ in rows], dtype=torch.int32)
        self.repetition = torch.tensor([rng.choice([1.0, 1.3, 0.7, 2.0]) for _ in rows])
        self.presence = torch.tensor([rng.choice([0.0, 0.6, -0.4]) for _ in rows])
        self.frequency = torch.tensor([rng.choice([0.0, 0.3, -0.2]) for _ in rows])
        self.bias_start = self.bias_ids = self.bias = self.mask = self.mask_row = None
        if biases:
            many = [rng.randint(0, biases) for _ in rows]
            self.bias_start = torch.tensor(np.concatenate([[0], np.cumsum(many)]), dtype=torch.int32)
            self.bias_ids = torch.randint(-1, min(vocab, 3 * biases) + 1, (sum(many) + 1,), generator=g, dtype=torch.int32)      # some twice, some no tokens
            self.bias = 4 * torch.randn(sum(many) + 1, generator=g)
        if masks:
            self.mask = torch.randint(-2 ** 31, 2 ** 31, (masks, (vocab + 31) // 32 + 1), generator=g, dtype=torch.int64).int()
            self.mask[0] = 0                                                # nothing is allowed
            self.mask_row = torch.randint(-2, masks + 2, (self.n,), generator=g, dtype=torch.int32)
        for name in without:
            setattr(self, name, None)

    def call(self, out=None, **kw):
        up = lambda t: None if t is None else t.cuda()  # noqa: E731
        z = self.logits.cuda() if out is None or not isinstance(out, str) else None
        if out == "in place":
            whole = torch.full((self.n, self.vocab + 5), 9.0, device="cuda").to(self.dtype)
            whole[:, :self.vocab] = self.logits.cuda()
            out = z = whole[:, :self.vocab]
        return binding.ppd_adjust_logits(z, up(self.row_start), **{k: up(getattr(self, k)) for k in RULES}, out=out, **kw)

    def exact(self):
        """(values, sizes that roundings are of) in 64 bits."""
        x = self.logits.double()
        size = x.abs()
        for s in range(len(self.rows)):
            lo, hi = int(self.row_start[s]), int(self.row_start[s + 1])
            for r in range(lo, hi):
                text = []
                if self.history is not None:
                    text += self.history[s, :int(self.history_len[s])].tolist()
                if self.ids is not None:
                    text += self.ids[lo:r + 1].tolist()
                prompt = max(0, int(self.prompt_len[s])) if self.prompt_len is not None else 0
                one = lambda t, d: d if t is None else float(t[s])  # noqa: E731
                rep, pre, fre = one(self.repetition, 1.0), one(self.presence, 0.0), one(self.frequency, 0.0)
                for t in set(text):
                    if 0 <= t < self.vocab:
                        n = text[prompt:].count(t)
                        if rep > 0:
                            x[r, t] = x[r, t] / rep if x[r, t] > 0 else x[r, t] * rep
                        size[r, t] = max(size[r, t], x[r, t].abs())
                        if n:
                            x[r, t] -= fre * n + pre
                            size[r, t] += abs(fre) * n + abs(pre)
                if self.bias is not None:
                    e = slice(int(self.bias_start[s]), int(self.bias_start[s + 1]))
                    for t, v in dict(zip(self.bias_ids[e].tolist(), self.bias[e].tolist())).items():
                        if 0 <= t < self.vocab:
                            x[r, t] += v
                            size[r, t] += abs(v)
                if self.mask is not None and 0 <= int(self.mask_row[r]) < len(self.mask):
                    bits = np.unpackbits(self.mask[int(self.mask_row[r])].numpy().view(np.uint8), bitorder="little")[:self.vocab]
                    x[r, torch.from_numpy(bits == 0)] = -math.inf
        return x, size

    def check(self, **kw):
        want, size = self.exact()
        for out in (None, torch.full((self.n, self.vocab), 7.0, device="cuda").to(self.dtype), "in place"):
            got = self.call(out, **kw)
            torch.cuda.synchronize()
            if out == "in place":
                assert (torch.as_strided(got, (self.n - 1, 5), (self.vocab + 5, 1), got.storage_offset() + self.vocab) == 9.0).all()      # (what lies behind a row)
            lo, hi = int(self.row_start[0]), int(self.row_start[-1])
            if out is not None:
                left = self.logits.cuda() if isinstance(out, str) else torch.full_like(got, 7.0)
                assert torch.equal(got[:lo], left[:lo]) and torch.equal(got[hi:], left[hi:])
            x, w, z = got[lo:hi].cpu().double(), want[lo:hi], size[lo:hi]
            assert torch.equal(torch.isinf(x), torch.isinf(w)) and not x.isnan().any()
            # the reciprocal and the product, the penalty's product and sum, two more sums: 6 roundings of fp32, then one to the type
            tol = 6 * 2.0 ** -24 * z + torch.nan_to_num(w.abs(), posinf=0.0) * HALF_STEP[self.dtype] * (1 + 2.0 ** -10) + TINY[self.dtype]
            bad = ((x - w).abs() > tol) & torch.isfinite(w)
            assert not bad.any(), (bad.nonzero()[:5], x[bad][:5], w[bad][:5])
            same = z == self.logits[lo:hi].double().abs()
            untouched = same & (w == self.logits[lo:hi].double())
            assert torch.equal(x[untouched], self.logits[lo:hi].double()[untouched])
        return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 7, 8, 33, 1000, 1025, 2049, 4096, 8200])
@pytest.mark.parametrize("rows", [[1], [4], [1, 3, 0, 7, 2]])
def test_types_and_vocabularies(dtype, vocab, rows):
    Case(rows, vocab, dtype, biases=6, masks=4, seed=vocab).check()
    Case(rows, vocab, dtype, biases=0, masks=0, seed=vocab + 1, pad=2).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ["ids", "prompt_len", "repetition", "presence", "frequency"])
def test_each_may_be_left_out(dtype, name):
    Case([1, 3, 0, 7, 2], 500, dtype, biases=4, masks=3, without=(name,)).check()


@pytest.mark.parametrize("without", [("history", "history_len"), ("bias", "bias_ids", "bias_start"), ("mask", "mask_row"), ("repetition", "presence", "frequency"),
                                     ("history", "history_len", "ids"), RULES])
def test_groups_may_be_left_out(without):
    Case([1, 3, 0, 7, 2], 500, F32, biases=4, masks=3, without=without).check()
    Case([1, 3, 0, 7, 2], 500, BF16, biases=4, masks=3, without=without, stride=501).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_many_workgroups(dtype):
    """The larger pieces of the vocabulary, and shares of rows."""
    Case([2] * 130, 16500, dtype, before=60, biases=9, masks=5).check()
    Case([70, 3, 40, 33], 70001, dtype, before=60, biases=9, masks=5, pad=1).check()


def test_long_sequences():
    Case([300], 900, F32, before=30).check()
    Case([0, 100, 1, 90], 2100, BF16, before=3000, biases=300, masks=2).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("stride", [0, 501, 503, 512])
def test_strides(dtype, stride):
    c = Case([1, 3, 2], 500, dtype, biases=5, masks=2, stride=stride, pad=3, start=2)
    want = c.check()
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    whole = torch.full((c.n, 511), 3.0, device="cuda").to(dtype)
    got = binding.ppd_adjust_logits(c.logits.cuda(), up(c.row_start), **{k: up(getattr(c, k)) for k in RULES}, out=whole[:, 4:504])
    assert torch.equal(got[2:8], want[2:8]) and (whole[:, :4] == 3.0).all() and (whole[:, 504:] == 3.0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_logits_that_are_no_numbers(dtype):
    """Infinities and NaN stay what they are, whatever is done beside them; a mask takes them, too."""
    c = Case([3], 100, dtype, before=0, masks=2)
    c.logits[:, 0], c.logits[:, 1], c.logits[:, 2], c.logits[:, 3] = math.inf, -math.inf, math.nan, -0.0
    c.history = torch.arange(0, 50, dtype=torch.int32)[None].repeat(1, 1)
    c.history_len, c.prompt_len, c.ids = torch.tensor([6], dtype=torch.int32), None, torch.tensor([7, 8, 9], dtype=torch.int32)
    c.mask[0], c.mask_row = 0, torch.tensor([-1, 0, 5], dtype=torch.int32)
    c.repetition, c.presence, c.frequency = torch.tensor([1.5]), torch.tensor([0.5]), torch.tensor([0.25])
    for out in (None, "in place"):
        got = c.call(out).cpu()
        for r in (0, 2):
            assert got[r, 0] == math.inf and got[r, 1] == -math.inf and got[r, 2].isnan() and float(got[r, 3]) == -0.75
        assert (got[1] == -math.inf).all()
    c.history_len[0] = 0
    assert torch.signbit(c.call().cpu()[0, 3])                     # what nothing is done to keeps its bits


@pytest.mark.parametrize("factor", [0.0, -1.0, math.nan])
def test_factors_that_are_none(factor):
    c = Case([2, 2], 300, F32)
    c.repetition[:] = factor
    c.check()


def test_lengths_and_numbers_outside_their_range():
    c = Case([2, 3, 1], 300, F32, biases=5, masks=3)
    good = c.call()
    c.history_len = torch.tensor([-5, 2 ** 31 - 1, 4], dtype=torch.int32)
    c.prompt_len = torch.tensor([2 ** 31 - 1, -2 ** 31, 4], dtype=torch.int32)
    c.call()
    c.history_len[1] = c.history.shape[1]
    c.history_len[0] = 0
    c.check()
    c.bias_start = torch.tensor([-9, 2 ** 31 - 1, -2 ** 31, 3], dtype=torch.int32)
    c.ids = torch.tensor([2 ** 31 - 1, -2 ** 31, 300, -1, 299, 5], dtype=torch.int32)
    c.call()
    torch.cuda.synchronize()
    for starts in ([0, 20, 10, 30], [30, 20, 10, 0], [0, 30, -7, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]):
        x = Case([2, 3, 1], 300, F32, biases=5, masks=3)
        x.row_start = torch.tensor(starts, dtype=torch.int32)
        whole = torch.full((10, 300), 7.0, device="cuda")
        x.call(whole[2:8])
        torch.cuda.synchronize()
        assert (whole[:2] == 7.0).all() and (whole[8:] == 7.0).all()
    assert good.shape == (6, 300)


def test_same_bits_every_time():
    c = Case([9, 1, 4], 3000, BF16, before=4000, biases=400, masks=3)
    first = c.call()
    for _ in range(5):
        assert torch.equal(c.call(), first)


def test_the_largest_vocabulary():
    Case([1, 2], 2 ** 24, BF16, biases=6, masks=2, seed=4).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_spread_unevenly(dtype):
    """A sequence with most of the rows, others with one or none, and more sequences than are looked at at once."""
    Case([1, 0, 77, 1, 0, 16, 17], 1500, dtype, before=30, biases=5, masks=3, seed=2, start=3, pad=2).check()
    rows = [0, 1] * 150 + [100] + [1, 2, 0] * 70
    Case(rows, 40, dtype, before=5, biases=2, masks=2, seed=3, pad=1).check()


def test_very_many_rows():
    """More runs of rows than a grid's second size."""
    n = 1200000
    z = torch.zeros(n, 3, device="cuda")
    start = torch.tensor([0, 5, 5, n - 7, n], dtype=torch.int32, device="cuda")
    bias = torch.tensor([1.0, 2.0, 3.0, 4.0], device="cuda")
    out = binding.ppd_adjust_logits(z, start, bias_start=torch.arange(5, dtype=torch.int32, device="cuda"), bias_ids=torch.tensor([0, 1, 2, 0], dtype=torch.int32, device="cuda"), bias=bias)
    want = torch.zeros_like(z)
    want[:5, 0], want[5:n - 7, 2], want[n - 7:, 0] = 1.0, 3.0, 4.0
    assert torch.equal(out, want)


def test_offsets_beyond_32_bits():
    n, vocab = 70000, 33000
    z = torch.zeros((n, vocab), dtype=BF16, device="cuda")
    z[n - 2:] = 2.0
    start = torch.tensor([0, n - 2, n], dtype=torch.int32, device="cuda")
    f = lambda *v: torch.tensor(v, device="cuda")  # noqa: E731
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    ids[n - 2], ids[n - 1] = 32999, 32998
    out = binding.ppd_adjust_logits(z, start, ids=ids, repetition=f(1.0, 2.0), presence=f(0.0, 0.25), out=z)
    torch.cuda.synchronize()
    assert out[n - 2, 32999] == 0.75 and out[n - 2, 32998] == 2.0 and out[n - 1, 32998] == 0.75 and out[n - 1, 32999] == 0.75 and out[n - 1, 0] == 2.0
    assert int((out[:n - 2] != 0).sum()) == 0


def test_streams_and_replays():
    c = Case([2, 3, 1], 2500, F32, before=30, biases=5, masks=3)
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    z, start, rest = c.logits.cuda(), c.row_start.cuda(), {k: up(getattr(c, k)) for k in RULES}
    ref = c.call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.ppd_adjust_logits(z, start, **rest, stream=side)
    side.synchronize()
    assert torch.equal(got, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = binding.ppd_adjust_logits(z, start, **rest)
    for i in range(3):
        z.copy_(torch.randn_like(z))
        rest["history_len"] += 1                                   # the replays follow the lengths
        rest["ids"].copy_(torch.randint(0, 2500, (6,)))
        graph.replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, binding.ppd_adjust_logits(z, start, **rest))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("masks", [0, 3])
def test_no_rows(dtype, masks):
    """Tensors without elements have no address."""
    c = Case([0, 0], 300, dtype, biases=4, masks=masks)
    assert c.n == 0
    for out in (None, torch.empty((0, 300), dtype=dtype, device="cuda"), "in place"):
        assert c.call(out).shape == (0, 300)
    assert Case([0], 1, dtype, without=RULES).call().shape == (0, 1)
    torch.cuda.synchronize()


def same_as_with(c, **inside):
    """The call's result, which is to the bit that of the same numbers inside their ranges, and that the definition's."""
    got = c.call()
    for name, values in inside.items():
        assert not torch.equal(getattr(c, name), torch.tensor(values, dtype=torch.int32))
        setattr(c, name, torch.tensor(values, dtype=torch.int32))
    assert torch.equal(got, c.check())


@pytest.mark.parametrize("dtype", TYPES)
def test_numbers_outside_their_range_count_as_the_next_inside(dtype):
    def case(**numbers):
        c = Case([2, 3, 1], 300, dtype, biases=5, masks=3, without=("mask", "mask_row"))
        c.repetition, c.presence, c.frequency = torch.tensor([1.5, 0.75, 2.0]), torch.tensor([0.5, -0.25, 1.0]), torch.tensor([0.25, 0.5, -0.125])
        for name, values in numbers.items():
            setattr(c, name, torch.tensor(values, dtype=torch.int32))
        return c

    whole = case().history.shape[1]
    many = case().bias.numel()
    same_as_with(case(history_len=[-5, 2 ** 31 - 1, -2 ** 31], prompt_len=[0, 3, 1]), history_len=[0, whole, 0])
    same_as_with(case(history_len=[whole, 7, whole], prompt_len=[2 ** 31 - 1, -2 ** 31, whole + 5]), prompt_len=[whole + 2, 0, whole + 1])
    same_as_with(case(history_len=[-1, whole + 1, 4], prompt_len=[2 ** 31 - 1, -2 ** 31, -1]), history_len=[0, whole, 4], prompt_len=[2, 0, 0])
    same_as_with(case(bias_start=[-9, 2 ** 31 - 1, -2 ** 31, 3]), bias_start=[0, many, 0, 3])
    same_as_with(case(bias_start=[-2 ** 31, 1, many + 1, 2 ** 31 - 1]), bias_start=[0, 1, many, many])
    c = case(ids=[2 ** 31 - 1, -2 ** 31, 300, -1, 299, 0])
    got = c.call()
    assert torch.equal(got, c.check())
    c.ids = torch.tensor([-1, -1, -1, -1, 299, 0], dtype=torch.int32)
    assert torch.equal(got, c.call())
