"""The token step as it is used: a toy speech-token model (one layer of random weights around the three operators) answers prompts of several sessions,
prompt by append and attend of many tokens, then token by token - launched one by one, and as one captured graph whose positions, tokens and random
numbers move on in device memory."""
import numpy as np
import pytest
import torch

from tests import token_util as tu
from tests.test_gpu_sample import pick

pytestmark = pytest.mark.gpu

D, H, HKV, VOCAB, SINK, WINDOW, EPS = 64, 8, 2, 1031, 3, 24, 1e-6


class Toy:
    def __init__(self, dc, prompts, steps, seed=0, dtype=torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
        n, self.dc, self.prompts, self.dtype = len(prompts), dc, prompts, dtype
        width = (H + 2 * HKV) * D
        self.embed, self.w_in, self.w_out = rand(VOCAB, 128).to(dtype), (rand(128, width) / 128 ** 0.5).to(dtype), (rand(H * D, VOCAB) / 8).to(dtype)
        self.norm = dc.QKNorm(1 + 0.1 * rand(D), 1 + 0.1 * rand(D), torch.tensor([500.0 ** (-j / 16) for j in range(16)], device="cuda"), eps=EPS)
        self.k, self.v = (torch.full((n + 1, HKV, SINK + WINDOW + max(prompts), D), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        self.cache = dc.TokenCache(self.k, self.v, H, n_sink=SINK, window=WINDOW)
        self.sessions = torch.randperm(n + 1, generator=g, device="cuda")[:n].to(torch.int32)
        self.u = torch.rand(steps, n, generator=g, device="cuda")
        self.rules = dict(temperature=0.7 + 0.1 * torch.arange(n, device="cuda"), top_k=torch.tensor([0, 40, 3, 0][:n], dtype=torch.int32, device="cuda"),
                          top_p=torch.full((n,), 0.9, device="cuda"), min_p=torch.full((n,), 0.01, device="cuda"))
        self.text = [torch.randint(VOCAB, (t,), generator=g, device="cuda") for t in prompts]

    def qkv(self, tokens):
        return self.embed[tokens.long()] @ self.w_in

    def prompt(self):
        cu = torch.tensor([0] + list(np.cumsum(self.prompts)), dtype=torch.int32, device="cuda")
        batch = self.dc.TokenBatch(self.sessions, torch.zeros(len(self.prompts), dtype=torch.int32, device="cuda"), cu, int(cu[-1]), max(self.prompts))
        x = self.qkv(torch.cat(self.text))
        out = self.cache.attend(self.cache.append(x, batch, self.norm), batch)
        return x, out, out[cu[1:].long() - 1]

    def step(self, tokens, batch, u, out_tokens, keep=None):
        """One token of every session: tokens -> the next ones, in out_tokens."""
        x = self.qkv(tokens)
        q = self.cache.append(x, batch, self.norm)
        o = self.cache.attend(q, batch)
        logits = o.flatten(1).float() @ self.w_out.float()
        self.dc.sample_tokens(logits, u, tokens=out_tokens, **self.rules)
        if keep is not None:
            keep.append((x, q, o, logits))


@pytest.fixture(scope="module")
def dc():
    import paper_2609_35115_b200 as dc
    dc.load_library()
    return dc


def test_answers_one_by_one_and_as_a_graph(dc):
    prompts, steps = [17, 40, 5, 61], 50
    n, seen, texts = len(prompts), [], []
    for captured in (False, True):
        toy = Toy(dc, prompts, steps)
        x, out, last = toy.prompt()
        tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
        dc.sample_tokens(last.flatten(1).float() @ toy.w_out.float(), toy.u[0], tokens=tokens, **toy.rules)
        start = torch.tensor(prompts, dtype=torch.int32, device="cuda")
        batch, u, text = dc.TokenBatch(toy.sessions, start), torch.empty(n, device="cuda"), [tokens.clone()]
        if captured:
            stream, graph, spare = torch.cuda.Stream(), torch.cuda.CUDAGraph(), (toy.k.clone(), toy.v.clone())
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                toy.step(tokens, batch, u.fill_(0.5), torch.empty_like(tokens))      # (warm-up: the products' library chooses its kernels)
            stream.synchronize()
            toy.k.copy_(spare[0])
            toy.v.copy_(spare[1])
            with torch.cuda.graph(graph, stream=stream):
                toy.step(tokens, batch, u, tokens)
                start += 1
        for t in range(1, steps):
            u.copy_(toy.u[t])
            if captured:
                graph.replay()
            else:
                toy.step(tokens, batch, u, tokens, seen)
                start += 1
            text.append(tokens.clone())
        toy.cache.check()
        texts.append(torch.stack(text))
        if not captured:
            first = (toy, x, out)
    assert torch.equal(texts[0], texts[1])
    assert len(set(texts[0].flatten().tolist())) > 20

    # every operator's part of it against 64 bits, on what it was given
    toy, x, out = first
    freq, gains = toy.norm._kept[2], toy.norm._kept[:2]
    at = 0
    history = []
    for i, t in enumerate(prompts):
        history.append([x[at:at + t]] + [s[0][i:i + 1] for s in seen])
        at += t
    for i, t in enumerate(prompts):
        rows = torch.cat(history[i]).double().view(-1, H + 2 * HKV, D)
        pos = torch.arange(len(rows), device="cuda")
        k64, size = tu.norm_rope(rows[:, H:H + HKV].clone(), gains[1], pos, freq, EPS, False)
        last = len(rows) - 1
        live = [p for p in range(len(rows)) if p < SINK or p > last - WINDOW]
        where = [tu.row_of(p, SINK, toy.k.shape[2] - SINK) for p in live]
        k = toy.k[toy.sessions[i].long()][:, where].transpose(0, 1).double()
        assert ((k - k64[live]).abs() <= tu.HALF[toy.dtype] * k64[live].abs() * 1.00001 + 24 * 2.0 ** -24 * size[live] + 1e-30).all()
        assert torch.equal(toy.v[toy.sessions[i].long()][:, where].transpose(0, 1), rows[live, H + HKV:].to(toy.dtype))
        q = seen[-1][1][i].double()[None]
        want, mag, worst = tu.attention(q, k.transpose(0, 1), rows[live, H + HKV:].transpose(0, 1), torch.tensor(live, device="cuda"), pos[-1:], SINK, WINDOW, D ** -0.5)
        assert ((seen[-1][2][i].double() - want[0]).abs() <= tu.attention_bound(want, mag, worst, len(live), D, toy.dtype, False)[0]).all()
    rules = {name: r.double().cpu().numpy() for name, r in toy.rules.items()}
    for t, (_, _, _, logits) in enumerate(seen):
        for i in range(n):
            want, _ = pick(logits[i].double().cpu().numpy(), float(toy.u[t + 1, i]), rules["temperature"][i], int(rules["top_k"][i]), rules["top_p"][i], rules["min_p"][i])
            assert int(texts[0][t + 1, i]) == want
