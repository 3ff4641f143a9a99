"""A decoder whose first layer drafts and whose layers together check the drafts, as a server would run it: ppd_paged_append and
ppd_paged_attention in every layer, ppd_early_topk behind the first, ppd_verify_drafts at the end.  The tokens have to be those that the
same model gives in 64 bits, one token after the other, from the whole sequence each time."""
import functools

import pytest
import torch

from paged_common import Batch
from paper_2307_05908_amd import binding

pytestmark = pytest.mark.gpu

D, HEADS, KV_HEADS, HD, FF, VOCAB, LAYERS, PAGE, DRAFTS, EPS, THETA = 128, 4, 2, 64, 256, 500, 2, 24, 2, 1e-5, 10000.0
PROMPTS = [[7, 3, 400, 12, 9], [250], list(range(60, 117))]
STEPS = 9


def weights():
    g = torch.Generator().manual_seed(12)

    def w(n, m, s=1.0):
        return torch.randn(n, m, generator=g) * s * m ** -0.5
    layers = []
    for i in range(LAYERS):
        s = 1.0 if i == 0 else 0.4                             # (so that the first layer is right now and then)
        layers.append(dict(q=w(HEADS * HD, D), k=w(KV_HEADS * HD, D), v=w(KV_HEADS * HD, D), o=w(D, HEADS * HD, s), up=w(FF, D), down=w(D, FF, s),
                           qg=1 + 0.1 * torch.randn(HD, generator=g), kg=1 + 0.1 * torch.randn(HD, generator=g)))
    return dict(layers=layers, emb=torch.randn(VOCAB, D, generator=g), gain=1 + 0.1 * torch.randn(D, generator=g), head=w(VOCAB, D, 2.0))


def each(m, f):
    return {k: [each(x, f) for x in v] if isinstance(v, list) else f(v) for k, v in m.items()}


def rms(x):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)


def layer64(w, x):
    """A layer over a whole sequence, in 64 bits."""
    n = x.shape[0]
    h = rms(x)
    q, k, v = ((h @ w[c].T).view(n, -1, HD) for c in "qkv")
    a = torch.arange(n, dtype=torch.float64)[:, None, None] * THETA ** (-2.0 * torch.arange(HD // 2, dtype=torch.float64) / HD)

    def turned(y, gain):
        y = rms(y) * gain
        lo, hi = y[..., :HD // 2], y[..., HD // 2:]
        return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)
    q, k = turned(q, w["qg"]), turned(k, w["kg"])
    z = torch.einsum("ihgd,jhd->hgij", q.view(n, KV_HEADS, -1, HD), k) * HD ** -0.5
    z = z.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -torch.inf)
    x = x + torch.einsum("hgij,jhd->ihgd", z.softmax(-1), v).reshape(n, -1) @ w["o"].T
    return x + torch.nn.functional.silu(rms(x) @ w["up"].T) @ w["down"].T


def best64(m, tokens, layers):
    """The model's next token, and by how much it leads."""
    x = m["emb"][torch.tensor(tokens)]
    for w in m["layers"][:layers]:
        x = layer64(w, x)
    z = (rms(x[-1]) * m["gain"]) @ m["head"].T
    top = z.topk(2)
    return int(top.indices[0]), float(top.values[0] - top.values[1])


@functools.lru_cache(maxsize=None)
def expected():
    """Per sequence: the tokens, and how many drafts each step takes."""
    m = each(weights(), lambda t: t.double())
    out = []
    for prompt in PROMPTS:
        seq, taken, least = list(prompt), [], 1e9
        for _ in range(STEPS):
            drafts = []
            for _ in range(DRAFTS):
                t, lead = best64(m, seq + drafts, 1)
                drafts.append(t)
                least = min(least, lead)
            n = 0
            while True:
                t, lead = best64(m, seq, LAYERS)
                least = min(least, lead)
                seq.append(t)
                if n == DRAFTS or drafts[n] != t:
                    break
                n += 1
            taken.append(n)
        # fp32 through two layers of sums of at most 256 products: thousands of roundings of 2^-24 at a size of some tens at most
        assert least > 2e-3, least
        out.append((seq[len(prompt):], taken))
    return out


class Server:
    def __init__(self):
        self.m = each(weights(), lambda t: t.cuda())
        n = len(PROMPTS)
        most = max(map(len, PROMPTS)) + STEPS * (DRAFTS + 1) + DRAFTS + 1
        per = -(-most // PAGE)
        g = torch.Generator().manual_seed(1)
        self.pages = torch.randperm(n * per, generator=g).int().view(n, per).cuda()
        self.cache = [torch.full((2, n * per, PAGE, KV_HEADS, HD), torch.nan, device="cuda") for _ in range(LAYERS)]

    def layers(self, ids, q_start, kv_len, count):
        x = self.m["emb"][ids.long()]
        for w, (kc, vc) in zip(self.m["layers"][:count], self.cache):
            h = rms(x)
            q, k, v = ((h @ w[c].T).view(len(ids), -1, HD) for c in "qkv")
            at = (kc, vc, self.pages, q_start, kv_len)
            q = binding.ppd_paged_append(*at, q, k, v, w["qg"], w["kg"], EPS, HD, THETA, q_out=q)
            o, _ = binding.ppd_paged_attention(q, *at)
            x = x + o.view(len(ids), -1) @ w["o"].T
            x = x + torch.nn.functional.silu(rms(x) @ w["up"].T) @ w["down"].T
        return x

    def logits(self, x):
        return (rms(x) * self.m["gain"]) @ self.m["head"].T

    def prompts(self):
        """All of the prompts but their last tokens, through all layers as one batch."""
        new = torch.tensor([0] + [len(p) - 1 for p in PROMPTS]).int()
        ids = torch.tensor([t for p in PROMPTS for t in p[:-1]]).int().cuda()
        self.layers(ids, new.cumsum(0).int().cuda(), new[1:].cuda(), LAYERS)
        self.length, self.last = new[1:].cuda(), torch.tensor([p[-1] for p in PROMPTS]).int().cuda()

    def drafts(self):
        """[n, 1 + DRAFTS]: the last tokens and what the first layer makes of them."""
        n, cols = len(PROMPTS), [self.last]
        for i in range(DRAFTS):
            x = self.layers(cols[-1], torch.arange(n + 1, dtype=torch.int32, device="cuda"), self.length + 1 + i, 1)
            cols.append(torch.cat([binding.ppd_early_topk(x[s], self.m["gain"], None, self.m["head"], 1, 1, EPS)[0] for s in range(n)]))
        return torch.stack(cols, 1)

    def check(self, ids, kv_len, temperature, uniform):
        n = len(PROMPTS)
        q_start = torch.arange(0, n * (DRAFTS + 1) + 1, DRAFTS + 1, dtype=torch.int32, device="cuda")
        z = self.logits(self.layers(ids.view(-1), q_start, kv_len, LAYERS))
        return binding.ppd_verify_drafts(z, ids.view(-1), q_start, uniform, temperature=temperature)

    def take(self, tokens, accepted):
        tokens = tokens.view(len(PROMPTS), DRAFTS + 1)
        self.length = self.length + accepted + 1                  # (what a draft that was not taken has left in the pages is written over)
        self.last = tokens.gather(1, accepted[:, None].long())[:, 0].contiguous()
        return [t[:a + 1] for t, a in zip(tokens.tolist(), accepted.tolist())]


def run(server, check):
    out, taken = [[] for _ in PROMPTS], [[] for _ in PROMPTS]
    for _ in range(STEPS):
        ids = server.drafts()
        tokens, accepted = check(ids, server.length + DRAFTS + 1)
        for s, got in enumerate(server.take(tokens, accepted)):
            out[s] += got
            taken[s].append(len(got) - 1)
    return out, taken


def greedy(n):
    return torch.zeros(n, device="cuda"), torch.full((n * (DRAFTS + 1), 2), 0.5, device="cuda")


def test_greedy_tokens_are_those_of_the_whole_model():
    want = expected()
    assert 0 < sum(map(sum, (t for _, t in want))) < DRAFTS * STEPS * len(PROMPTS)      # some are taken, some are not
    server = Server()
    server.prompts()
    rules = greedy(len(PROMPTS))
    out, taken = run(server, lambda ids, kv: server.check(ids, kv, *rules))
    for s, (tokens, counts) in enumerate(want):
        assert out[s] == tokens and taken[s] == counts


def test_the_checking_step_as_a_graph():
    want = expected()
    server = Server()
    server.prompts()
    rules = greedy(len(PROMPTS))
    ids, kv = server.drafts(), server.length + DRAFTS + 1
    server.check(ids, kv, *rules)                                 # (libraries are loaded outside of the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tokens, accepted = server.check(ids, kv, *rules)

    def check(new_ids, new_kv):
        ids.copy_(new_ids)
        kv.copy_(new_kv)
        graph.replay()
        return tokens.clone(), accepted.clone()
    out, taken = run(server, check)
    for s, (t, counts) in enumerate(want):
        assert out[s] == t and taken[s] == counts


def test_sampled_tokens_are_the_same_on_two_streams_at_once():
    """Two servers with random numbers of their own, each on its stream, give what each gives alone."""
    def numbers(seed):
        g = torch.Generator().manual_seed(seed)
        return [torch.rand(len(PROMPTS) * (DRAFTS + 1), 2, generator=g).cuda() for _ in range(STEPS)]
    t = torch.tensor([0.7, 1.0, 0.0], device="cuda")

    def steps(server, us):
        for u in us:
            tokens, accepted = server.check(server.drafts(), server.length + DRAFTS + 1, t, u)
            yield server.take(tokens, accepted)
    alone = []
    for seed in (1, 2):
        server = Server()
        server.prompts()
        alone.append(list(steps(server, numbers(seed))))
    assert alone[0] != alone[1]
    servers, sides, runs, got = [Server(), Server()], [torch.cuda.Stream(), torch.cuda.Stream()], [], [[], []]
    us = [numbers(1), numbers(2)]
    torch.cuda.synchronize()
    for server, side, u in zip(servers, sides, us):
        with torch.cuda.stream(side):
            server.prompts()
            runs.append(steps(server, u))
    for _ in range(STEPS):
        for side, r, g in zip(sides, runs, got):
            with torch.cuda.stream(side):
                g.append(next(r))
    assert got == alone


def test_scratch_memory_that_is_not_in_a_row_is_refused():
    b = Batch([1, 2], [3000, 90], 4, 2, 128, torch.bfloat16).cuda()
    thin = torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 26)
    with pytest.raises(ValueError, match="workspace"):
        binding.ppd_paged_attention(b.q, b.k_cache, b.v_cache, b.pages, b.q_start, b.kv_len, workspace=thin)
    with pytest.raises(ValueError, match="workspace"):
        binding.ppd_verify_drafts(torch.zeros(3, 100, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"),
                                  torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.zeros(3, 2, device="cuda"), workspace=thin)
