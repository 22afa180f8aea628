"""The serving operators together, as a server uses them: a PT model whose layers run on a paged cache, with requests that come
and go, prompts in chunks beside decode steps, a sequence forked in the middle of a page, pages compacted, and sampled
tokens.  Every logit is compared with the oracle's run of that request alone, and every token with the definition."""
import numpy as np
import pytest

from oracle import pt_oracle as O
from paper_2602_07306_amd import inputs as I
from tests import serving_reference as R
from tests.helpers import BF16_TOL, FP32_TOL, assert_close, small_bf16_config

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PAGE = 16


class Server:
    """A PT model in torch products around the paged operators; the tracks' heads lie side by side in the cache."""

    def __init__(self, cfg, W, n_pages):
        from paper_2602_07306_amd import binding as PB
        self.PB, self.cfg = PB, cfg
        self.ty = torch.bfloat16 if cfg.dtype == I.PT_BF16 else torch.float32
        dev = lambda a: torch.as_tensor(np.asarray(a, dtype=np.float32)).cuda()
        self.W = {n: [[dev(W[n][t, l]) for l in range(cfg.n_layers)] for t in range(cfg.n_tracks)] for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2")}
        self.embed, self.head, self.gf = dev(W["embed"]), dev(W["head"]), dev(W["gf"])
        heads = cfg.n_tracks * cfg.n_kv_heads
        self.k, self.v = (torch.full((cfg.n_layers, n_pages, heads, PAGE, cfg.head_dim), float("nan"), dtype=self.ty, device="cuda") for _ in range(2))
        self.cache = PB.PTPagedCache(self.k, self.v)
        self.rope = PB.PTRope(PB.PT_ROPE_HALF, cfg.head_dim, cfg.rope_theta)
        self.free = list(range(n_pages))[::-1]
        self.pages, self.len = {}, {}
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def norm(self, x, g):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.cfg.rms_eps) * g

    def step(self, work):
        """work: {request: new tokens}.  Returns {request: logits of its last row}."""
        cfg, PB = self.cfg, self.PB
        for r, toks in work.items():
            self.len[r] = self.len.get(r, 0) + len(toks)
            own = self.pages.setdefault(r, [])
            while len(own) * PAGE < self.len[r]:
                own.append(self.free.pop())
        names = list(work)
        n = [len(work[r]) for r in names]
        start = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        table = np.zeros((len(names), max(len(self.pages[r]) for r in names)), dtype=np.int32)
        for b, r in enumerate(names):
            table[b, :len(self.pages[r])] = self.pages[r]
        dev = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda()
        batch = PB.PTPagedBatch(dev(start), dev([self.len[r] for r in names]), dev(table), total_rows=int(start[-1]), max_q_len=max(n),
                                max_kv_len=max(self.len[r] for r in names), status=self.status)
        x = self.embed[dev(np.concatenate([work[r] for r in names])).long()]
        T, hd = cfg.n_tracks, cfg.head_dim
        h = [x] * T
        for l in range(cfg.n_layers):
            a = [self.norm(h[t], self.W["g1"][t][l]) for t in range(T)]
            heads = lambda w: torch.cat([(a[t] @ self.W[w][t][l]).view(x.shape[0], -1, hd) for t in range(T)], dim=1).to(self.ty)
            q = PB.pt_paged_append(self.cache, l, batch, heads("wk"), heads("wv"), q=heads("wq"), rope=self.rope)
            o = PB.pt_paged_attention(self.cache, l, batch, q).float().chunk(T, dim=1)
            h = [h[t] + o[t].reshape(x.shape[0], -1) @ self.W["wo"][t][l] for t in range(T)]
            for t in range(T):
                m = self.norm(h[t], self.W["g2"][t][l])
                h[t] = h[t] + (torch.nn.functional.silu(m @ self.W["wg"][t][l]) * (m @ self.W["wu"][t][l])) @ self.W["wd"][t][l]
            if (l + 1) % cfg.block_depth == 0:
                merged = PB.pt_track_merge([t.contiguous() for t in h], cfg.merge_scale)
                h = [merged] * T
        last = torch.from_numpy(start[1:].astype(np.int64) - 1).cuda()
        logits = (self.norm(h[0][last], self.gf) @ self.head).contiguous()
        return dict(zip(names, logits)), logits

    def fork(self, old, new):
        """Whole pages are shared; the last, unfinished one is copied."""
        own = list(self.pages[old])
        if self.len[old] % PAGE:
            fresh = self.free.pop()
            self.PB.pt_page_copy(self.cache, [(own[-1], fresh)])
            own[-1] = fresh
        self.pages[new], self.len[new] = own, self.len[old]

    def drop(self, r):
        shared = {p for o, ps in self.pages.items() if o != r for p in ps}
        self.free += [p for p in self.pages.pop(r) if p not in shared]
        del self.len[r]

    def compact(self):
        """Moves the used pages to the front of the pool; what lies behind is free (and overwritten here)."""
        used = sorted({p for ps in self.pages.values() for p in ps})
        holes = [p for p in range(len(used)) if p not in used]
        far = [p for p in used if p >= len(used)]
        to = dict(zip(far, holes))
        self.PB.pt_page_copy(self.cache, list(to.items()))
        self.pages = {r: [to.get(p, p) for p in ps] for r, ps in self.pages.items()}
        self.k[:, len(used):] = float("nan")
        self.v[:, len(used):] = float("nan")
        self.free = list(range(len(used), self.k.shape[1]))[::-1]


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_a_server_equals_every_request_alone(kind):
    cfg = (I.PTConfig(n_tracks=2, n_layers=4, block_depth=2, d_model=128, n_heads=4, n_kv_heads=2, head_dim=32, d_ffn=256, vocab=512, max_batch=1,
                      max_seq=160, dtype=I.PT_F32) if kind == "fp32" else small_bf16_config(n_kv_heads=1, max_seq=160, max_batch=1))
    tol = FP32_TOL if kind == "fp32" else BF16_TOL
    W = I.make_weights(cfg, 21)
    s = Server(cfg, W, 60)
    rng = np.random.default_rng(22)
    prompt = {r: I.make_tokens(23 + i, 1, n, cfg.vocab)[0] for i, (r, n) in enumerate((("a", 70), ("b", 3), ("c", 33), ("d", 16)))}
    given = {}          # tokens a request has seen

    def check(work):
        byname, logits = s.step(work)
        for r, t in work.items():
            given[r] = np.concatenate([given.get(r, np.zeros(0, np.int32)), t]).astype(np.int32)
        got = logits.cpu().numpy()
        for i, r in enumerate(work):
            st = O.PTState(cfg, 1, cfg.max_seq)
            want = O.pt_prefill(cfg, W, st, tokens=given[r][None])["logits"][0, -1]
            assert_close(got[i][None], want[None], tol, "%s after %d" % (r, len(given[r])))
        n = len(work)
        u = rng.random(n).astype(np.float32)
        T, k, p = rng.uniform(0.5, 1.2, n).astype(np.float32), rng.choice([0, 5, 40], n).astype(np.int32), rng.choice([1.0, 0.9], n).astype(np.float32)
        dev = lambda a: torch.from_numpy(a).cuda()
        tok = s.PB.pt_sample(logits, dev(u), dev(T), dev(k), dev(p)).cpu().numpy()
        assert tok.tolist() == [R.sample(got[i], u[i], float(T[i]), int(k[i]), float(p[i])) for i in range(n)]
        return {r: tok[i:i + 1] for i, r in enumerate(work)}

    nxt = check({"a": prompt["a"][:40], "b": prompt["b"]})              # two prompts, the first in chunks
    nxt = {**nxt, **check({"b": nxt["b"], "a": prompt["a"][40:], "c": prompt["c"]})}   # a decode step beside chunks
    for _ in range(3):
        nxt = check({r: nxt[r] for r in ("c", "a", "b")})
    s.fork("a", "a2")                                                   # in the middle of a page
    given["a2"] = given["a"].copy()
    nxt["a2"] = (nxt["a"] + 1) % cfg.vocab
    nxt = check({r: nxt[r] for r in ("a", "a2", "b", "c")})
    s.drop("c")
    s.drop("a")                                                         # its whole pages live on in the fork
    s.compact()
    nxt = {**nxt, **check({"a2": nxt["a2"], "d": prompt["d"], "b": nxt["b"]})}
    for _ in range(3):
        nxt = check({r: nxt[r] for r in ("d", "b", "a2")})
    assert int(s.status) == 0


def test_sampled_generation_of_a_model():
    """pt_sample in the place of the greedy choice, between the decode steps of a handle."""
    from paper_2602_07306_amd import binding as PB
    cfg = small_bf16_config(max_batch=3)
    m = PB.PTModel(cfg)
    m.pt_init_weights(31)
    tokens = torch.from_numpy(I.make_tokens(31, 3, 20, cfg.vocab)).cuda()
    logits, _ = m.pt_prefill(tokens)
    T, k, p, q = (torch.full((3,), v, dtype=t, device="cuda") for v, t in ((0.8, torch.float32), (50, torch.int32), (0.9, torch.float32), (0.01, torch.float32)))
    gen = torch.Generator(device="cuda").manual_seed(5)
    for _ in range(5):
        u = torch.rand(3, generator=gen, device="cuda")
        tok = PB.pt_sample(logits, u, T, k, p, q)
        x, us = logits.cpu().numpy(), u.cpu().numpy()
        assert tok.tolist() == [R.sample(x[i], us[i], float(np.float32(0.8)), 50, float(np.float32(0.9)), float(np.float32(0.01))) for i in range(3)]
        logits, _, _ = m.pt_decode_step(tok)
    m.pt_sync_status()
    m.close()
