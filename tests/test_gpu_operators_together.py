"""The 4-bit LM head, the sampling controls, the verification and the cache pages one after the other, as a decode cycle uses them."""
import numpy as np
import pytest
import torch

from oracle import oracle as orc
from paper_2510_26527_b200 import binding, buildlib, staged, synth
from tests import plain_operators as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    buildlib.build()
    binding.load_library()
    orc.build()
    assert torch.cuda.is_available()


class Cycle:
    """One level of a chain for B sequences: both models' 4-bit heads, controls, verification, pages."""

    def __init__(self, B, k, V, d, seed):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.B, self.k, self.V = B, k, V
        self.hp = torch.randn((B, k + 1, d), generator=g).to(torch.bfloat16)
        self.hq = (self.hp[:, :k].float() + 0.3 * torch.randn((B, k, d), generator=g)).to(torch.bfloat16)
        self.codes = torch.randint(0, 16, (V, d), generator=g, dtype=torch.uint8)
        self.scales = (torch.rand((V, d // 128), generator=g) * 0.01 + 0.01).to(torch.bfloat16)
        self.zero = torch.randint(6, 10, (V, d // 128), generator=g, dtype=torch.uint8)
        self.kw = {"history": rng.integers(0, V, (B, 40)).astype(np.int32), "repetition": np.full(B, 1.2, np.float32),
                   "frequency": np.full(B, 0.3, np.float32), "presence": np.full(B, 0.2, np.float32),
                   "draft_tokens": rng.integers(0, V, (B, k)).astype(np.int32)}
        self.allowed = rng.random((B, k + 1, V)) < 0.7
        np.put_along_axis(self.allowed[:, :k], self.kw["draft_tokens"][..., None], True, 2)
        self.u = torch.from_numpy(synth.philox_uniforms(seed, 1, B, k + 1)[0]).contiguous()
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
        self.d = {n: dev(x) for n, x in self.kw.items()}
        self.masks = [dev(plain.mask_words(self.allowed)), dev(plain.mask_words(self.allowed[:, :k]))]
        self.q = binding.polyspec_pack_quantized(self.codes.to(DEV))
        self.s, self.z = self.scales.to(DEV), self.zero.to(DEV)
        self.h = [self.hp.to(DEV).reshape(-1, d), self.hq.to(DEV).reshape(-1, d)]
        self.rows = [k + 1, k]
        self.logits = [torch.empty((B * r, V), device=DEV) for r in self.rows]
        self.ws = torch.empty(binding.polyspec_verify_level_workspace(B, k, V, binding.F32), dtype=torch.uint8, device=DEV)
        self.out = {"accepted_len": torch.empty(B, dtype=torch.int32, device=DEV), "next_token": torch.empty(B, dtype=torch.int32, device=DEV)}
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.pages = binding.CachePages.new(B, 16, 16 * B, 4, DEV)
        self.len = torch.full((B,), 13, dtype=torch.int32, device=DEV)
        binding.polyspec_cache_reserve(self.pages, self.len)
        self.ud = self.u.to(DEV)

    def run(self):
        binding.polyspec_cache_reserve(self.pages, self.len, plus=self.k, device_status=self.status)
        for h, out, r, mask in zip(self.h, self.logits, self.rows, self.masks):
            binding.polyspec_lm_head_quantized(h, self.q, self.s, self.z, out=out, device_status=self.status)
            block = out.view(self.B, r, self.V)
            binding.polyspec_process_logits(block, **self.d, mask=mask, out=block, device_status=self.status)
        p, q = (x.view(self.B, r, self.V) for x, r in zip(self.logits, self.rows))
        binding.polyspec_verify_level(p, q, self.d["draft_tokens"], self.ud, 0.9, workspace=self.ws, out=self.out, device_status=self.status)
        binding.polyspec_cache_rollback(self.pages, self.len, self.out["accepted_len"], device_status=self.status)

    def check(self):
        torch.cuda.synchronize()
        assert int(self.status) == 0
        d = self.codes.shape[1]
        for h, out, r in zip((self.hp, self.hq), self.logits, self.rows):
            raw, size = plain.head(h.reshape(-1, d), self.codes, self.scales, self.zero)
            raw, size = raw.view(self.B, r, self.V).numpy(), size.view(self.B, r, self.V).numpy()
            want, _, more = plain.controls(raw, allowed=self.allowed[:, :r], **{("draft" if n == "draft_tokens" else n): v for n, v in self.kw.items()})
            got = out.view(self.B, r, self.V).cpu().double().numpy()
            # the head's bound, which the penalty (a factor of at most 1.2) carries on, and the controls' own
            tol = 1.2 * (128 + d // 128) * 2.0 ** -23 * size + 4 * 2.0 ** -24 * (more + np.abs(raw))
            finite = np.isfinite(want)
            assert (np.isneginf(got) == ~finite).all()
            # where a logit is so near zero that its sign is not sure, the penalty multiplies or divides: |z| (r - 1/r) more
            assert (np.abs(np.where(finite, got - np.where(finite, want, 0), 0)) <= tol * 1.5).all()
        p, q = (x.view(self.B, r, self.V).cpu() for x, r in zip(self.logits, self.rows))
        ora = orc.verify_level(p, q, torch.from_numpy(self.kw["draft_tokens"]), self.u, 0.9)
        assert (self.out["accepted_len"].cpu().numpy() == ora["accepted_len"]).all()
        assert (self.out["next_token"].cpu().numpy() == ora["next_token"]).all()
        assert (self.pages.len.cpu().numpy() == 13 + ora["accepted_len"]).all()
        assert all(self.allowed[b, a, t] for b, (a, t) in enumerate(zip(ora["accepted_len"], ora["next_token"])))


@pytest.mark.parametrize("B,k,V,d", [(1, 3, 1024, 256), (6, 4, 2048, 512), (20, 7, 4096, 256)])
def test_cycle(B, k, V, d):
    c = Cycle(B, k, V, d, seed=B)
    c.run()
    c.check()


def test_cycle_captured():
    c = Cycle(5, 4, 2048, 256, seed=3)
    c.run()                                 # workspaces exist
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for x in c.logits:
        x.zero_()
    graph.replay()
    c.check()


def _staged(B, N, V, K, mu, ntok, caches=None):
    g = torch.Generator(device=DEV).manual_seed(5)
    M1 = torch.randn((B, N, V), generator=g, device=DEV) * 2
    M2 = M1 + 0.5 * torch.randn((B, N, V), generator=g, device=DEV)
    M3 = M1 + torch.randn((B, N, V), generator=g, device=DEV)
    drafts = torch.multinomial(torch.softmax(M3, -1).reshape(B * N, V), 1, generator=g).reshape(B, N).to(torch.int32).contiguous()
    u2 = torch.from_numpy(synth.philox_uniforms(6, B, 60, K + 1)).to(DEV)
    u1 = torch.from_numpy(synth.philox_uniforms(7, B, 40, staged.MAX_BLOCK + 1)).to(DEV)
    return staged.StagedBatch(M1, M2, M3, drafts, u2, u1, K, mu, ntok, 1.0, caches)


@pytest.mark.parametrize("P", [1, 4, 16])
def test_staged_loop_keeps_its_page_tables_in_step(P):
    B, N, V, K, mu, ntok = 5, 80, 256, 3, 5, 30
    plainly = _staged(B, N, V, K, mu, ntok).run()
    most = (N + K + P) // P + 1
    caches = {m: (binding.CachePages.new(B, most, B * most, P, DEV), []) for m in ("M1", "M2", "M3")}
    loop = _staged(B, N, V, K, mu, ntok, caches)
    while int(loop.state["remaining"]):
        before = {m: c.len.clone() for m, (c, _) in caches.items()}
        loop.iteration()
        torch.cuda.synchronize()
        assert int(loop.status) == 0
        t, cnt = loop.state["t"], loop.state["cnt"]
        for m, (c, _) in caches.items():
            length, table, refs = c.len.cpu(), c.table.cpu(), c.refs.cpu()
            # never more than stands but for the last token emitted; at least what stood before, up to that
            assert (length <= (t + cnt - 1).clamp(min=0).cpu()).all(), m
            assert (length >= torch.minimum(before[m], (t + cnt - 1).clamp(min=0)).cpu()).all(), m
            held = (length + P - 1) // P
            assert ((table >= 0).sum(1) == held).all()
            assert refs.sum() == held.sum() and refs.max() <= 1
        # M_2 has been given everything that stands but the last token, unless M_1 has just added one
        assert (caches["M2"][0].len >= t + cnt - 2).all()
    got = loop.results()
    for key in ("committed", "n_committed", "cycles", "per_cycle"):
        assert torch.equal(got[key], plainly[key])


def test_staged_loop_reports_a_pool_too_small():
    caches = {"M2": (binding.CachePages.new(5, 30, 3, 4, DEV), [])}
    loop = _staged(5, 80, 256, 3, 5, 30, caches)
    for _ in range(4):
        loop.iteration()
    torch.cuda.synchronize()
    assert int(loop.status) == binding.ERR_NO_PAGES
    with pytest.raises(ValueError):
        _staged(5, 80, 256, 3, 5, 30, {"M2": (binding.CachePages.new(4, 30, 3, 4, DEV), [])})
    with pytest.raises(ValueError):
        _staged(5, 80, 256, 3, 5, 30, {"M4": (binding.CachePages.new(5, 30, 3, 4, DEV), [])})


def _with_caches(loop, B, N, K, P=4):
    most = (N + K + P) // P + 1
    loop.caches = {m: (binding.CachePages.new(B, most, B * most, P, DEV), []) for m in ("M1", "M2", "M3")}
    return {m: c for m, (c, _) in loop.caches.items()}


def test_staged_loop_leaves_the_pages_of_a_model_that_sits_out():
    """M_1's table stands still in every iteration in which its pass is not due."""
    B, N, V, K, mu = 6, 120, 256, 3, 9
    loop = _staged(B, N, V, K, mu, 50)
    pages = _with_caches(loop, B, N, K)
    waited = 0
    while int(loop.state["remaining"]):
        before = pages["M1"].len.tolist()
        loop.iteration()
        after, due = pages["M1"].len.tolist(), loop.block_len1.tolist()
        for b in range(B):
            if not due[b]:
                assert after[b] == before[b], (b, before, after)
                waited += 1
        assert int(loop.status) == 0
    assert waited > 3 * B


@pytest.mark.parametrize("K,mu", [(1, 4), (3, 5), (5, 1)])
def test_staged_loop_lengths_are_the_tokens_each_model_was_given(K, mu):
    """What a model was given, counted from the positions of its passes: rows p .. p + n of a pass take the tokens before p + n.
    A length is as many of those as still stand, the last token emitted never among them."""
    B, N, V = 6, 120, 256
    loop = _staged(B, N, V, K, mu, 40)
    loop.M3.copy_(loop.M2)                                  # q = p: M_2 accepts every draft
    pages = _with_caches(loop, B, N, K)
    want = {m: [0] * B for m in pages}
    whole = 0
    while int(loop.state["remaining"]):
        loop.iteration()
        torch.cuda.synchronize()
        pos2, len2, pos1, len1 = (x.tolist() for x in (loop.pos2, loop.block_len2, loop.pos1, loop.block_len1))
        stands = [max(t + c - 1, 0) for t, c in zip(loop.state["t"].tolist(), loop.state["cnt"].tolist())]
        whole += sum(a == K for a, n in zip(loop.out2["accepted_len"].tolist(), len2) if n)
        for b in range(B):
            # M_3 drafts the K tokens (its last draft is not given back to it), M_2 scores K + 1 rows, M_1 len1 + 1 rows
            given = {"M3": pos2[b] + K - 1 if len2[b] else 0, "M2": pos2[b] + K if len2[b] else 0, "M1": pos1[b] + len1[b] if len1[b] else 0}
            for m in want:
                want[m][b] = min(max(want[m][b], given[m]), stands[b])
        for m, c in pages.items():
            assert c.len.tolist() == want[m], m
    assert whole > B and int(loop.status) == 0


def test_staged_loop_sequences_out_of_the_loop_take_no_pages():
    """Finished sequences keep their tables as they are; one that fails in its first round, or never had a round, holds nothing."""
    B, N, V, K, mu = 5, 80, 256, 6, 1
    loop = _staged(B, N, V, K, mu, 2)
    loop.M2[3, : K + 1] = float("nan")
    pages = _with_caches(loop, B, N, K)
    done = [0] * B
    for _ in range(12):
        before = {m: c.len.tolist() for m, c in pages.items()}
        loop.iteration()
        for m, c in pages.items():
            now = c.len.tolist()
            assert [n for n, d in zip(now, done) if d] == [n for n, d in zip(before[m], done) if d], m
        done = loop.state["done"].tolist()
    assert all(done)
    for c in pages.values():
        assert int(c.len[3]) == 0 and int((c.table[3] >= 0).sum()) == 0
        assert int(c.refs.sum()) == int(((c.len + 3) // 4).sum())
    short = _staged(B, K, V, K, mu, 2)                      # a block and its bonus row do not fit into K positions
    pages = _with_caches(short, B, K, K)
    short.iteration()
    assert all(short.state["done"].tolist())
    assert all(int(c.len.abs().sum()) == 0 and int(c.refs.abs().sum()) == 0 for c in pages.values())
