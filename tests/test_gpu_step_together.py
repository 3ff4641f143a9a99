"""A server's step that checks drafts, with keys and values of 4 bits, as one: ppd_paged_plan, then ppd_paged_append_fp4 and ppd_paged_attention_fp4
in every layer, ppd_adjust_logits, ppd_verify_drafts, and the next plan from what was accepted.  The host reads nothing between the steps: conversations
come and go, and one of them waits for pages.  Each operator is held to its definition at what the others gave it, and a captured step to an eager one."""
import threading

import numpy as np
import pytest
import torch

from fp4_common import NAMES, Batch4, quantised64, values64
from paged_common import append64, attention64
from paper_2307_05908_amd import binding
from test_gpu_adjust import Case
from test_gpu_append_fp4 import EPS
from test_gpu_attention_fp4 import limits
from test_gpu_plan import rule as plan_rule
from test_gpu_verify_drafts import rule as verify_rule

pytestmark = pytest.mark.gpu

D, HEADS, KV_HEADS, HD, FF, VOCAB, LAYERS, PAGE, DRAFTS, THETA = 128, 4, 2, 64, 256, 500, 2, 8, 2, 10000.0
SEQS, MOST, N_PAGES, ROWS = 4, 96, 15, 64
PROMPTS = {0: [7, 3, 400, 12, 9], 1: [250, 251], 2: list(range(60, 107)), 3: [5] * 30}
SECOND = {2: [9, 8, 7, 6, 5, 4]}            # sequence 2's next conversation
END, STEPS = 6, 14


class Server:
    def __init__(self, dtype, seed=3):
        g = torch.Generator().manual_seed(12)

        def w(n, m, s=1.0):
            return (torch.randn(n, m, generator=g) * s * m ** -0.5).to(dtype).cuda()

        def gain(n):
            return (1 + 0.1 * torch.randn(n, generator=g)).to(dtype).cuda()
        self.layers = [dict(q=w(HEADS * HD, D), k=w(KV_HEADS * HD, D), v=w(KV_HEADS * HD, D), o=w(D, HEADS * HD, 0.4), up=w(FF, D), down=w(D, FF, 0.4), qg=gain(HD),
                            kg=gain(HD)) for _ in range(LAYERS)]
        self.emb, self.head = w(VOCAB, D, D ** 0.5), w(VOCAB, D, 2.0)

        def ints(*x, dtype=torch.int32):
            return torch.tensor(x, dtype=dtype, device="cuda")
        self.pages, self.ring = torch.full((SEQS, MOST // PAGE), -1, dtype=torch.int32, device="cuda"), torch.randperm(N_PAGES, generator=g).int().cuda()
        self.counters, self.held, self.kept = ints(0, N_PAGES, dtype=torch.int64), ints(*[0] * SEQS), ints(*[0] * SEQS)
        self.wanted, self.prompt_len = ints(*[0] * SEQS), ints(*[0] * SEQS)
        self.uniform = torch.zeros(ROWS, 2, device="cuda")
        self.temperature = torch.tensor([0.0, 0.9, 1.3, 0.7], device="cuda")
        self.texts = torch.zeros(SEQS * MOST + 1, dtype=torch.int32, device="cuda")         # (and a place for what is no token)
        self.repetition, self.presence = torch.tensor([1.0, 1.3, 0.8, 1.0], device="cuda"), torch.tensor([0.0, 0.2, 0.0, -0.5], device="cuda")
        self.frequency = torch.tensor([0.0, 0.1, 0.4, 0.0], device="cuda")
        self.bias_start, self.bias_ids = ints(0, 2, 2, 3, 3), ints(7, 9, 250)
        self.bias = torch.tensor([-float("inf"), 1.5, 2.0], device="cuda")
        odd = ints(*[0xaaaaaaaa - 2 ** 32] * ((VOCAB + 31) // 32))
        self.mask = torch.stack([odd, ~odd])
        self.grammar = ints(-1, -1, 0, 1)                                                   # of each sequence
        self.cache = []
        for _ in range(LAYERS):
            shape = (N_PAGES, PAGE, KV_HEADS)
            self.cache.append([torch.full((*shape, x), y, dtype=torch.uint8, device="cuda") for x, y in ((HD // 2, 0x77), (HD // 32, 255)) * 2])
        self.follows = (self.emb.float() @ self.head.float().T).argmax(1).int()             # what is drafted behind a token: what the model without its layers gives
        self.numbers = torch.Generator().manual_seed(seed)
        self.seen = None                                                                    # a list, if the operators' inputs and outputs are wanted
        self.at = 0

    def note(self, name, **what):
        if self.seen is not None:
            self.seen.append((name, {k: [x.cpu() for x in v] if isinstance(v, list) else None if v is None else v.cpu() for k, v in what.items()}))

    def text(self):
        return self.texts[:-1].view(SEQS, MOST)

    def forward(self, plan):
        ids = torch.where(plan.row_seq < 0, 0, self.texts[(plan.row_seq.clamp(min=0) * MOST + plan.positions.clamp(min=0)).long()])
        x = self.emb[ids.long()]
        x = torch.where(plan.row_seq[:, None] < 0, 0, x)
        for w, pool in zip(self.layers, self.cache):
            h = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            q, k, v = ((h @ w[c].T).view(ROWS, -1, HD) for c in "qkv")
            where = (*(pool[i] for i in (0, 1, 2, 3)), self.pages, plan.q_start, plan.kv_len)
            before = [t.clone() for t in pool] if self.seen is not None else None
            out, _, _ = binding.ppd_paged_append_fp4(*where, q, k, v, w["qg"], w["kg"], EPS, HD, THETA)
            self.note("append", q=q, k=k, v=v, out=out, before=before, after=pool, qg=w["qg"], kg=w["kg"], pages=self.pages, **plan._asdict())
            o, lse = binding.ppd_paged_attention_fp4(out, *where, out=torch.zeros_like(q), want_lse=True)
            self.note("attention", q=out, out=o, lse=lse, pool=pool, pages=self.pages, **plan._asdict())
            x = x + o.view(ROWS, -1) @ w["o"].T
            h = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            x = x + torch.nn.functional.silu(h @ w["up"].T) @ w["down"].T
        return ids, x @ self.head.T

    def planned(self):
        self.note("plan before", pages=self.pages, ring=self.ring, counters=self.counters, held=self.held, kept=self.kept, wanted=self.wanted)
        plan = binding.ppd_paged_plan(self.pages, self.ring, self.counters, self.held, self.wanted, PAGE, ROWS, kept=self.kept, kv_len=self.held, counters_out=self.counters)
        self.note("plan", pages=self.pages, ring=self.ring, **plan._asdict())
        return plan

    def prompts(self):
        """All of a prompt but its last token; those that have no room wait."""
        plan = self.planned()
        self.forward(plan)
        self.kept.copy_(self.held)

    def step(self):
        """The last token and its drafts through the model; the tokens that it gave (-1: none) and how many drafts were taken."""
        plan = self.planned()
        base = plan.kv_len - plan.granted                                                   # the last token's position
        first = torch.arange(SEQS, device="cuda") * MOST + base
        for i in range(DRAFTS):
            self.texts[first + i + 1] = self.follows[self.texts[first + i].long()]
        ids, z = self.forward(plan)
        rows = torch.where(plan.row_seq < 0, -1, self.grammar[plan.row_seq.clamp(min=0).long()])
        rules = dict(ids=ids, history=self.text(), history_len=base, prompt_len=self.prompt_len, repetition=self.repetition, presence=self.presence,
                     frequency=self.frequency, bias_start=self.bias_start, bias_ids=self.bias_ids, bias=self.bias, mask=self.mask, mask_row=rows)
        was = z.clone()
        binding.ppd_adjust_logits(z, plan.q_start, **rules, out=z)
        self.note("adjust", logits=was, out=z, row_start=plan.q_start, granted=plan.granted, **rules)
        tokens, accepted = binding.ppd_verify_drafts(z, ids, plan.q_start, self.uniform, temperature=self.temperature, tokens=torch.full_like(ids, -1))
        self.note("verify", z=z, ids=ids, granted=plan.granted, tokens=tokens, accepted=accepted, uniform=self.uniform, temperature=self.temperature)
        at = torch.where((tokens < 0) | (plan.row_seq < 0), SEQS * MOST, plan.row_seq * MOST + plan.positions + 1)
        self.texts[at.long()] = tokens
        self.kept.copy_(base + torch.where(plan.granted > 0, accepted + 1, 0))
        return plan.row_seq, tokens, accepted, plan.granted

    def admit(self, prompts):
        """New conversations; those that are there keep what they have."""
        self.wanted.zero_()
        for s, p in prompts.items():
            self.text()[s, :len(p)] = torch.tensor(p, dtype=torch.int32, device="cuda")
            self.prompt_len[s], self.kept[s], self.wanted[s] = len(p), 0, len(p) - 1

    def run(self, step=None):
        """Every step's tokens, sequence by sequence."""
        step, out = step or self.step, []
        self.admit({s: PROMPTS[s] for s in (0, 1, 2)})
        self.prompts()
        living = [0, 1, 2]
        for i in range(STEPS):
            if i == 1:
                self.admit({3: PROMPTS[3]})
                self.prompts()
                living.append(3)
            if i == END:                                                                    # its pages go to those who wait; it comes again with another prompt
                self.admit({})
                self.kept[2] = 0
                self.prompts()
                self.admit(SECOND)
                self.prompts()
            self.wanted.copy_(torch.tensor([(1 + DRAFTS) * (s in living) for s in range(SEQS)], dtype=torch.int32))
            self.uniform.copy_(torch.rand(ROWS, 2, generator=self.numbers))
            out.append([t.clone() for t in step()])
        torch.cuda.synchronize()
        return [[t.tolist() for t in o] for o in out]


def batch_of(c, dtype, pool=None):
    """The batch that an operator got, for its definition in 64 bits."""
    b = object.__new__(Batch4)
    new = c["granted"].tolist()
    b.__dict__ = dict(new=new, kv=c["kv_len"].tolist(), heads=HEADS, kv_heads=KV_HEADS, hd=HD, dtype=dtype, page=PAGE, rows=sum(new), n=ROWS, n_pages=N_PAGES,
                      pages=c["pages"], q=c["q"], k=c.get("k"), v=c.get("v"))
    if pool is not None:
        b.k_codes, b.k_scales, b.v_codes, b.v_scales = pool
        b.renew()
    return b


def hold(name, c, dtype, last):
    if name == "plan":
        want = plan_rule(last["pages"].tolist(), last["ring"].tolist(), last["counters"].tolist(), last["held"].tolist(), last["kept"].tolist(),
                         last["wanted"].tolist(), PAGE, ROWS)
        for k, x in want.items():
            assert c[k].tolist() == x, k
    elif name == "append":
        b = batch_of(c, dtype)
        (q, q_size), (k, _), place = append64(b, c["qg"], c["kg"], EPS, HD, THETA)
        (kc, ks), (vc, vs) = quantised64(k), quantised64(b.v[:b.rows])
        want = dict(zip(("k_codes", "k_scales", "v_codes", "v_scales"), c["before"]))
        for i, (_, slot) in enumerate(place):
            want["k_codes"][slot], want["k_scales"][slot], want["v_codes"][slot], want["v_scales"][slot] = kc[i], ks[i], vc[i], vs[i]
        assert sorted(want) == sorted(NAMES)
        for x, y in zip(c["after"], want.values()):
            assert torch.equal(x, y)
    elif name == "attention":
        b = batch_of(c, dtype, c["pool"])
        out, lse, size, reach = attention64(b)
        tol, ltol = limits(b, out, lse, size, reach)
        r = b.rows
        assert ((c["out"][:r].double() - out[:r]).abs() <= tol[:r]).all() and ((c["lse"][:r].double() - lse[:r]).abs() <= ltol[:r]).all()
        assert (c["out"][r:] == 0).all()
    elif name == "adjust":
        e = object.__new__(Case)
        e.__dict__ = dict(c, rows=c["granted"].tolist(), vocab=VOCAB, dtype=dtype, n=ROWS)
        want, size = e.exact()
        r = sum(e.rows)
        x, w, z = c["out"][:r].double(), want[:r], size[:r]
        # 6 roundings of fp32: the reciprocal and the product, the penalty's product and sum, two more sums; then one to the type
        step = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[dtype]
        tol = 6 * 2.0 ** -24 * z + torch.nan_to_num(w.abs(), posinf=0.0) * step * (1 + 2.0 ** -10) + 2.0 ** -133
        gone = torch.isinf(w)
        assert torch.equal(torch.isinf(x), gone) and ((x - w).abs()[~gone] <= tol[~gone]).all()
        assert torch.equal(c["out"][r:], c["logits"][r:])
    elif name == "verify":
        n = c["granted"].tolist()
        tokens, accepted, near = verify_rule([m - 1 for m in n], c["ids"].numpy(), c["z"].float().numpy(), None, c["temperature"].double().numpy(),
                                             c["uniform"].double().numpy())
        assert near > 2.0 ** -35, "the numbers are at a border"
        np.testing.assert_array_equal(c["tokens"][:sum(n)].numpy(), tokens)
        np.testing.assert_array_equal(c["accepted"].numpy(), accepted)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_operator_holds_at_what_the_others_give_it(dtype):
    server = Server(dtype)
    server.seen = []
    steps = server.run()
    last, names = None, []
    for name, c in server.seen:
        hold(name, c, dtype, last)
        last = c
        names.append(name)
    assert all(names.count(x) for x in ("plan", "append", "attention", "adjust", "verify"))
    taken, granted = np.array([s[2] for s in steps]), np.array([s[3] for s in steps])
    assert 0 < taken.sum() < DRAFTS * SEQS * STEPS
    assert (granted.sum(0) > 0).all() and (granted[1:] == 0).any()                         # all had their turn, some had to wait
    # a page belongs to one sequence, or is free
    held, pages, ring, (head, tail) = server.held.tolist(), server.pages.tolist(), server.ring.tolist(), server.counters.tolist()
    mine = [p for s in range(SEQS) for p in pages[s][:-(-held[s] // PAGE)]]
    assert sorted(mine + [ring[i % N_PAGES] for i in range(head, tail)]) == list(range(N_PAGES))


def graph_of(server):
    """A step as a graph.  (It runs once before, where no sequence asks for anything, so that libraries are loaded outside of the capture.)"""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        server.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = server.step()

    def step():
        graph.replay()
        return out
    return step


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_captured_step_gives_the_same_tokens(dtype):
    want = Server(dtype).run()
    server = Server(dtype)
    assert server.run(graph_of(server)) == want


def test_two_captured_steps_on_two_streams_at_once():
    want = [Server(torch.bfloat16, seed).run() for seed in (5, 6)]
    assert want[0] != want[1]
    servers, sides = [Server(torch.bfloat16, seed) for seed in (5, 6)], [torch.cuda.Stream() for _ in range(2)]
    steps = [graph_of(s) for s in servers]
    torch.cuda.synchronize()
    got, turn = [None, None], threading.Barrier(2)

    def run(i):
        def step():
            turn.wait(30)                                                                   # (their steps go out at the same time)
            return steps[i]()
        with torch.cuda.stream(sides[i]):
            got[i] = servers[i].run(step)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert got == want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_a_step_in_which_nobody_has_a_row(dtype):
    """Every operator takes the batch that the plan makes of it, and leaves the pages as they were."""
    def ints(*x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    pages, counters = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), torch.tensor([0, 9], device="cuda")
    plan = binding.ppd_paged_plan(pages, torch.arange(9, dtype=torch.int32, device="cuda"), counters, ints(0, 0), ints(0, 3), PAGE, 0)
    assert plan.q_start.tolist() == [0, 0, 0] and plan.granted.tolist() == [0, 0] and plan.counters.tolist() == [0, 9] and plan.slots.shape == (0,)
    pool = [torch.full((9, PAGE, KV_HEADS, x), 3, dtype=torch.uint8, device="cuda") for x in (HD // 2, HD // 32) * 2]
    where = (*pool, pages, plan.q_start, plan.kv_len)
    q, k, z = (torch.empty(0, *shape, dtype=dtype, device="cuda") for shape in ((HEADS, HD), (KV_HEADS, HD), (VOCAB,)))
    q, *values = binding.ppd_paged_append_fp4(*where, q, k, k.clone(), rotary_dim=HD, want_values=True)
    out, lse = binding.ppd_paged_attention_fp4(q, *where, want_lse=True)
    assert q.shape == out.shape == (0, HEADS, HD) and all(x.shape == (0, KV_HEADS, HD) for x in values) and lse.shape == (0, HEADS)
    mask = torch.full((1, (VOCAB + 31) // 32), -1, dtype=torch.int32, device="cuda")
    for rules in ({}, dict(repetition=torch.ones(2, device="cuda")), dict(mask=mask, mask_row=ints())):
        assert binding.ppd_adjust_logits(z, plan.q_start, ids=ints(), **rules).shape == (0, VOCAB)
    tokens, accepted = binding.ppd_verify_drafts(z, ints(), plan.q_start, torch.empty(0, 2, device="cuda"))
    torch.cuda.synchronize()
    assert tokens.shape == (0,) and accepted.shape == (2,) and all((t == 3).all() for t in pool)
