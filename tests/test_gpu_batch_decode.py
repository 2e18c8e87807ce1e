"""The operators together, as a server uses them: requests behind one shared prefix take their prompts
in, verify draft trees and roll back, layer by layer with torch's products between the operators, against
the library's own single-sequence passes on every request's whole sequence.

Both sides round the same activations to bf16 and sum in other orders: the logits are held to the
passes' own bar against the float64 model (2e-2 absolute, 1e-2 in the 2-norm), once for each side."""

import numpy as np
import pytest
import torch

import workloads

pytestmark = pytest.mark.gpu

P = 100


class Model:
    """A decoder forward over a batch's rows: torch's fp32 products, the library's operators between."""

    def __init__(self, shape, gen):
        self.s = shape
        f = lambda t: t.float()  # noqa: E731
        self.embed, self.final, self.head = f(gen.tok_embed()), f(gen.final_norm()), f(gen.lm_head())
        self.layers = [{k: f(v) for k, v in gen.layer(l).items()} for l in range(shape.n_layers)]

    def norm(self, x, g):
        return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.s.rms_eps) * g).to(torch.bfloat16)

    def forward(self, batch, tokens):
        s, N = self.s, tokens.shape[0]
        x = self.embed[tokens.long()]
        q = torch.zeros(N, s.n_heads, s.head_dim, dtype=torch.bfloat16, device="cuda")
        out = torch.zeros_like(q)
        for l, w in enumerate(self.layers):
            qkv = (self.norm(x, w["attn_norm"]).float() @ w["w_qkv"].t()).to(torch.bfloat16).view(N, 3 * s.n_heads, s.head_dim)
            batch.store(l, qkv[:, :s.n_heads], qkv[:, s.n_heads:2 * s.n_heads], qkv[:, 2 * s.n_heads:], q)
            batch.attention(l, q, out)
            x = x + out.view(N, -1).float() @ w["w_o"].t()
            gate, up = (self.norm(x, w["ffn_norm"]).float() @ w["w_gate_up"].t()).chunk(2, -1)
            x = x + (torch.nn.functional.silu(gate) * up).to(torch.bfloat16).float() @ w["w_down"].t()
        return self.norm(x, self.final).float() @ self.head.t()


@pytest.fixture(scope="module", params=["tiny", "wide"])
def model(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2309_04255_amd import binding

    shape = {"tiny": workloads.MODELS["tiny"],
             "wide": workloads.ModelShape("wide", 2, 512, 4, 128, 1000, 1998, seed=0x5EED0128)}[request.param]
    sess = binding.Session(shape, capacity=P + 300, max_n=128)
    gen = workloads.make_weights(shape, "cuda", gain_jitter=0.1)
    sess.load_weights(gen)
    return binding, shape, sess, Model(shape, gen)


def _near(got, want):
    got, want = got.double(), want.double()
    assert float((got - want).abs().max()) <= 4e-2
    assert float((got - want).norm() / want.norm()) <= 2e-2


def test_requests_behind_one_prefix(model):
    binding, shape, sess, net = model
    rng = np.random.default_rng(11)
    prefix = workloads.draw_tokens(P, shape.vocab, seed=3)
    sess.prefill(prefix, 0)
    k_prefix, v_prefix = sess.k_cache.clone(), sess.v_cache.clone()  # (the session goes on as the reference)
    B, N = 4, 160
    batch = binding.Batch(shape, B, N, n_pages=16, max_pages=4, prefix_len=P, k_cache=k_prefix, v_cache=v_prefix)
    # what each request holds behind the prefix, and its next rows: first its prompt, then trees
    seqs = [[] for _ in range(B)]
    prompts = [workloads.draw_tokens(m, shape.vocab, seed=20 + i) for i, m in enumerate((60, 1, 64, 17))]
    rows = [(np.asarray(p), workloads.chain_tree(len(p))) for p in prompts]
    for step in range(4):
        start = np.concatenate([[0], np.cumsum([len(t) for t, _ in rows])]).astype(np.int32)
        tokens, parent = np.zeros(N, np.int32), np.zeros(N, np.int32)
        for b, (t, p) in enumerate(rows):
            tokens[start[b]:start[b + 1]], parent[start[b]:start[b + 1]] = t, p
        dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        batch.plan(dev(start), dev([len(s) for s in seqs]), dev(parent))
        assert not batch.status.any()
        logits = net.forward(batch, dev(tokens))
        batch.advance()
        row_of = dev([start[b] + max(int(p), 0) for b, (t, par) in enumerate(rows) for p in par])
        given = torch.tensor(tokens[:start[B]], device="cuda")
        total = int(start[B])
        scores = binding.token_scores(logits[:total], given, 3, row_of=row_of)
        # the library's own pass over every request's sequence
        path, accept = np.full(N, -1, np.int32), np.zeros(B, np.int32)
        for b, (t, par) in enumerate(rows):
            if len(seqs[b]):
                sess.prefill(np.asarray(seqs[b]), P)
            n = sess.verify_tree(P + len(seqs[b]), t, par)
            want, _, _, _ = sess.results(n)
            mine = logits[start[b]:start[b + 1]]
            _near(mine.cpu(), want)
            ref = torch.log_softmax(mine.double(), -1)
            lp = scores["logprob"][start[b]:start[b + 1]].double()
            pick = torch.tensor(np.maximum(par, 0)).cuda()
            assert torch.allclose(lp, ref[pick, torch.tensor(t).cuda().long()], atol=1e-5)
            tree = sess.score_tree(t, par, 3)
            assert float(tree["logprob"][0]) == 0.0
            assert torch.allclose(tree["logprob"][1:].double(), lp[1:], atol=4e-2)
            # accept the whole prompt, later the branch of some node
            i = len(t) - 1 if step == 0 else int(rng.integers(len(t)))
            branch = []
            while i >= 0:
                branch.append(i)
                i = int(par[i])
            branch = branch[::-1]
            path[start[b]:start[b] + len(branch)] = branch
            accept[b] = len(branch) - 1
            seqs[b] += [int(t[i]) for i in branch]
        batch.commit(dev(path), dev(accept))
        rows = []
        for b in range(B):  # the next trees; a request that sits a step out
            par = workloads.random_tree(int(rng.integers(1, 24)), 4, seed=step * 10 + b)
            rows.append((workloads.draw_tokens(len(par), shape.vocab, seed=100 + step * 10 + b), par))
        if step == 1:
            keep = len(batch.free_pages)
            batch.release(1)  # the second request ends, another begins in its place
            assert len(batch.free_pages) > keep
            seqs[1] = []


def test_session_scores_a_text(model):
    binding, shape, sess, _ = model
    text = workloads.draw_tokens(200, shape.vocab, seed=5)  # (two chunks of the session's passes)
    sess.prefill(text[:10], 0)
    got = sess.score(text[10:], 10, k=4)
    rows = []
    for i in (0, 1, 126, 127, 128, 188, 189):
        sess.prefill(text[:11 + i], 0, want_logits=True)
        lp = torch.log_softmax(sess.last_logits.double(), -1)
        if i < 189:
            assert abs(float(got["logprob"][i]) - float(lp[int(text[11 + i])])) <= 4e-2
        else:
            assert float(got["logprob"][i]) == 0.0
        assert abs(float(got["entropy"][i]) - float(-(lp.exp() * lp).sum())) <= 4e-2
        assert abs(float(got["top_logprob"][i, 0]) - float(lp.max())) <= 4e-2
        rows.append(i)
    assert got["logprob"].shape == (190,) and got["top_token"].shape == (190, 4)
