"""The paged operators as they are used together: prompts admitted, beams forked,
tokens appended, attended to and selected over many steps, each hypothesis against
its own history; the same step recorded as a graph; other streams."""
import numpy as np
import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu


class Beams:
    """Device state of a beam search: two sets of tables, one pool per layer."""

    def __init__(self, kind, B, W, L, H, Hkv, hd, ps, V, max_len, layout, seed, n_pages=None):
        import torch

        from paged_common import CODE, DT, make_pool
        from paper_2503_17707_amd import binding as pb

        self.pb, self.torch = pb, torch
        self.B, self.W, self.L, self.H, self.Hkv, self.hd, self.ps, self.V = B, W, L, H, Hkv, hd, ps, V
        self.code, self.dt, R = CODE[kind], DT[kind], B * W
        self.width = -(-max_len // ps)
        self.n_pages = n_pages or R * self.width
        self.pool = make_pool(seed, kind, (L, self.n_pages), Hkv, ps, hd, layout)
        self.pool.fill_(float("nan"))
        i32 = dict(dtype=torch.int32, device="cuda")
        self.sets = [dict(tables=torch.full((R, self.width), -1, **i32), start=torch.zeros(R, **i32),
                          lens=torch.zeros(R, **i32), refs=torch.zeros(self.n_pages, **i32)) for _ in range(2)]
        self.short = torch.zeros(2, **i32)
        self.parents, self.tokens, self.alive = (torch.zeros(B, W, **i32) for _ in range(3))
        self.scores = torch.zeros(B, W, device="cuda")
        self.logits = torch.zeros(R, V, device="cuda")
        self.qkv = torch.zeros(L, R, (H + 2 * Hkv) * hd, dtype=self.dt, device="cuda")
        self.out = torch.zeros(L, R, H, hd, dtype=self.dt, device="cuda")
        need = max(pb.page_fork_workspace(R, self.n_pages), pb.beam_select_workspace(B, W, V),
                   pb.paged_attention_workspace(R, H, self.pool[0], self.width))
        self.ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")

    def split(self, l):
        a, b = self.H * self.hd, (self.H + self.Hkv) * self.hd
        x = self.qkv[l]
        return [x[:, i:j].unflatten(1, (-1, self.hd)) for i, j in ((0, a), (a, b), (b, x.shape[1]))]

    def step(self, i, eos):
        """Fork set i into the other one, append, attend, select."""
        pb, a, b = self.pb, self.sets[i], self.sets[1 - i]
        pb.op_page_fork(self.code, self.pool, self.parents.view(-1), a["tables"], a["lens"], a["refs"], self.alive.view(-1),
                        b["tables"], b["start"], b["lens"], b["refs"], self.short, self.ws)
        for l in range(self.L):
            q, k, v = self.split(l)
            pb.op_kv_append(self.code, k, v, self.pool[l], b["tables"], b["start"], b["lens"])
            pb.op_paged_attention(self.code, q, self.pool[l], b["tables"], b["lens"], self.out[l], scale=self.hd ** -0.5,
                                  workspace=self.ws, shared=True)
        pb.op_beam_select(self.logits, self.scores, self.alive, self.scores, self.tokens, self.parents, self.alive, eos=eos,
                          pad=0, workspace=self.ws)

    def admit(self, prompts, prompt_kv):
        """Prompts' pages for rows 0 .. B-1 of set 0, their keys and values, and beams on them."""
        torch, pb, B, W, R = self.torch, self.pb, self.B, self.W, self.B * self.W
        i32 = dict(dtype=torch.int32, device="cuda")
        lens = torch.tensor(prompts, **i32)
        one = dict(tables=torch.full((B, self.width), -1, **i32), start=torch.zeros(B, **i32), lens=torch.zeros(B, **i32),
                   refs=torch.zeros(self.n_pages, **i32))
        pb.op_page_fork(self.code, self.pool, torch.arange(B, **i32), torch.full((B, self.width), -1, **i32),
                        torch.zeros(B, **i32), torch.zeros(self.n_pages, **i32), lens, one["tables"], one["start"],
                        one["lens"], one["refs"], self.short, self.ws)
        assert self.short.tolist() == [0, 0] and one["lens"].tolist() == list(prompts)
        row0 = torch.tensor(np.concatenate([[0], np.cumsum(prompts)[:-1]]), **i32)
        for l in range(self.L):
            k, v = prompt_kv[l]
            pb.op_kv_append(self.code, k, v, self.pool[l], one["tables"], one["start"], one["lens"], row0=row0)
        s = self.sets[0]
        pb.op_page_fork(self.code, self.pool, torch.arange(R, **i32) // W, one["tables"], one["lens"], one["refs"],
                        torch.zeros(R, **i32), s["tables"], s["start"], s["lens"], s["refs"], self.short, self.ws)
        self.parents.copy_(torch.arange(R, **i32).view(B, W))
        self.alive.fill_(1)
        self.scores.fill_(-float("inf"))
        self.scores[:, 0] = 0


def _kv(torch, g, dt, rows, Hkv, hd):
    return [torch.randn((rows, Hkv, hd), generator=g).to(dt).cuda() for _ in range(2)]


@pytest.mark.parametrize("kind,layout,B,W,L,H,Hkv,hd,ps,prompts", [
    ("f16", "rows", 2, 4, 2, 4, 2, 64, 8, (5, 19)),
    ("bf16", "heads", 3, 3, 1, 6, 6, 128, 16, (16, 1, 31)),
    ("f16", "gaps", 1, 8, 2, 16, 1, 64, 5, (23,)),
])
def test_beam_search_against_histories(kind, layout, B, W, L, H, Hkv, hd, ps, prompts):
    import torch

    from paged_common import attention64, select64

    log("beam search", kind, layout, B, W, L, H, Hkv, hd, ps, prompts)
    V, eos, R, steps = 61, 2, B * W, 24
    s = Beams(kind, B, W, L, H, Hkv, hd, ps, V, max(prompts) + steps + 1, layout, 1)
    g = torch.Generator().manual_seed(7)
    prompt_kv = [_kv(torch, g, s.dt, sum(prompts), Hkv, hd) for _ in range(L)]
    s.admit(prompts, prompt_kv)
    # per hypothesis and layer its own keys and values
    begin = np.concatenate([[0], np.cumsum(prompts)])
    hist = [[torch.stack(prompt_kv[l], 1).cpu()[begin[r // W]:begin[r // W + 1]] for l in range(L)] for r in range(R)]
    alive, parents = np.ones((B, W), np.int32), np.arange(R)
    scores = s.scores.cpu().numpy()
    for step in range(steps):
        s.qkv.copy_(torch.randn(s.qkv.shape, generator=g))
        s.logits.copy_(torch.randn(s.logits.shape, generator=g) * 2)
        if step > 2:
            s.logits[:, eos] += 1.5
        new = [[torch.stack([x[r] for x in s.split(l)[1:]]).cpu() for l in range(L)] for r in range(R)]
        grows = alive.reshape(-1).copy()
        s.step(step % 2, eos)
        hist = [[torch.cat([hist[parents[r]][l], new[r][l][None]]) if grows[r] else hist[parents[r]][l] for l in range(L)]
                if parents[r] >= 0 else [torch.zeros(0, 2, Hkv, hd, dtype=s.dt)] * L for r in range(R)]
        now = s.sets[1 - step % 2]
        assert s.short.tolist() == [0, 0]
        tables, lens = now["tables"].cpu().numpy(), now["lens"].tolist()
        assert lens == [len(h[0]) for h in hist]
        held = tables[tables >= 0]
        assert np.array_equal(np.bincount(held, minlength=s.n_pages), now["refs"].cpu().numpy())
        for l in range(L):
            pages = s.pool[l].cpu()
            for r in range(R):  # bit for bit what the hypothesis went through
                got = [pages[tables[r, x // ps], :, :, x % ps] for x in range(lens[r])]
                assert not lens[r] or torch.equal(torch.stack(got), hist[r][l]), (step, l, r)
            ref, tol = attention64(s.split(l)[0], s.pool[l], tables, lens, ps, hd ** -0.5, 0)
            assert torch.all((s.out[l].double().cpu() - ref).abs() <= tol)
        want = select64(s.logits.cpu().numpy(), scores, alive, eos, 0)
        scores, alive = s.scores.cpu().numpy(), s.alive.cpu().numpy()
        assert np.array_equal(s.tokens.cpu().numpy(), want[1]) and np.array_equal(s.parents.cpu().numpy(), want[2])
        assert np.array_equal(alive, want[3])
        parents = s.parents.cpu().numpy().reshape(-1)
    log("  alive at the end", alive.tolist())


def test_recorded_step_equals_eager():
    """Two steps (set 0 to 1 and back) as one graph, replayed with new inputs and eager
    work in between, against the same steps run one by one; two graphs share the workspace."""
    import torch

    from paper_2503_17707_amd import binding as pb  # noqa: F401

    log("recorded beam step")
    prompts, L, eos = (40, 700), 2, 2
    args = ("f16", 2, 4, L, 8, 2, 64, 16, 3000, 780, "heads", 3)
    a, b = Beams(*args), Beams(*args)
    g = torch.Generator().manual_seed(9)
    prompt_kv = [_kv(torch, g, a.dt, sum(prompts), a.Hkv, a.hd) for _ in range(L)]
    a.admit(prompts, prompt_kv)
    b.admit(prompts, prompt_kv)
    side = torch.cuda.Stream()

    def fill(s, i):
        gg = torch.Generator(device="cuda").manual_seed(100 + i)
        s.qkv.copy_(torch.randn(s.qkv.shape, generator=gg, device="cuda"))
        s.logits.copy_(torch.randn(s.logits.shape, generator=gg, device="cuda") * 2)

    # both run one warm step pair eagerly, then b records
    for s in (a, b):
        fill(s, 0)
        s.step(0, eos)
        s.step(1, eos)
    keep = [x.clone() for x in (b.scores, b.alive, b.parents, b.tokens)]
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for i, gr in enumerate(graphs):
        with torch.cuda.graph(gr):
            b.step(i, eos)
    for x, y in zip((b.scores, b.alive, b.parents, b.tokens), keep):
        assert torch.equal(x, y)  # recording ran nothing
    for i in range(1, 13):
        fill(a, i)
        fill(b, i)
        a.step(0, eos)
        a.step(1, eos)
        if i % 3 == 0:  # on another stream
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                graphs[0].replay()
                graphs[1].replay()
            torch.cuda.current_stream().wait_stream(side)
        else:
            graphs[0].replay()
            graphs[1].replay()
        torch.cuda.synchronize()
        for name in ("scores", "alive", "parents", "tokens", "short"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (i, name)
        live = a.sets[0]["lens"].tolist()
        assert b.sets[0]["lens"].tolist() == live
        for n in ("tables", "refs", "start"):
            assert torch.equal(a.sets[0][n], b.sets[0][n]), (i, n)
        rows = [r for r in range(8) if live[r]]
        assert torch.equal(a.out[:, rows], b.out[:, rows])
    assert max(live) > 700


@pytest.mark.parametrize("dtype,hd", [("f16", 64), ("bf16", 128)])
def test_a_decoder_over_pages_matches_the_oracle(dtype, hd):
    """Prompts of two lengths and three tokens more, layer by layer through the single-kernel entry
    points, the cache in pages: each step's logits and tokens are the oracle's of the prompt so far."""
    import torch

    import oracle
    import synth
    from gpu_common import compare
    from paper_2503_17707_amd import binding as pb

    log("decoder over pages", dtype, hd)
    w = synth.Workload(name="paged", seed=51, n_layers=2, d_model=256, n_heads=256 // hd, d_ffn=512, vocab=900, max_pos=64,
                       dtype=dtype, batch=2, seq_len=29, n_adapters=0)
    code, dt = (pb.PB_F16, torch.float16) if dtype == "f16" else (pb.PB_BF16, torch.bfloat16)
    d, H, L = 256, 256 // hd, 2
    get = lambda l, n: torch.from_numpy(synth.base_tensor(w, l, n, dtype).view(np.int16)).view(dt).cuda()  # noqa: E731
    G = {n: get(-1, n) for n in synth.GLOBAL_TENSORS}
    layers = [{n: get(l, n) for n in synth.LAYER_TENSORS} for l in range(L)]
    for x in layers:
        x["wqkv"], x["bqkv"] = torch.cat([x["wq"], x["wk"], x["wv"]]), torch.cat([x["bq"], x["bk"], x["bv"]])
    lens, ps, n_pages, B = [12, 29], 16, 7, 2
    i32 = dict(dtype=torch.int32, device="cuda")
    pools = torch.full((L, n_pages, ps, 2, H, hd), float("nan"), dtype=dt, device="cuda").permute(0, 1, 3, 4, 2, 5)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    state = [torch.full((B, 4), -1, **i32), torch.zeros(B, **i32), torch.zeros(n_pages, **i32)]  # tables, lens, refs

    def forward(rows, grow, attend):
        """Appends rows [n, d] of new tokens (fp32), sequence after sequence; their last hidden states."""
        new = [torch.empty((B, 4), **i32), torch.empty(B, **i32), torch.empty(n_pages, **i32)]
        start, short = torch.empty(B, **i32), torch.empty(2, **i32)
        pb.op_page_fork(code, pools, torch.arange(B, **i32), *state, torch.tensor(grow, **i32), new[0], start, new[1], new[2],
                        short, ws)
        assert short.tolist() == [0, 0]
        state[:] = new
        n, row0 = len(rows), torch.tensor([0, grow[0]], **i32)
        h, a = torch.empty((n, d), dtype=dt, device="cuda"), torch.empty((n, d), dtype=dt, device="cuda")
        qkv, f = torch.empty((n, 3 * d), dtype=dt, device="cuda"), torch.empty((n, 512), dtype=dt, device="cuda")
        for l, x in enumerate(layers):
            pb.op_layernorm(code, rows, x["ln1_g"], x["ln1_b"], h)
            pb.op_gemm(code, 0, h, x["wqkv"], x["bqkv"], C=qkv, qscale=hd ** -0.5, qcols=d)
            q, k, v = (qkv[:, i * d:(i + 1) * d].unflatten(1, (H, hd)) for i in range(3))
            pb.op_kv_append(code, k, v, pools[l], state[0], start, state[1], row0=row0)
            attend(l, qkv, q, a)
            pb.op_gemm(code, 2, a, x["wo"], x["bo"], R=rows)
            pb.op_layernorm(code, rows, x["ln2_g"], x["ln2_b"], h)
            pb.op_gemm(code, 1, h, x["w1"], x["b1"], C=f)
            pb.op_gemm(code, 2, f, x["w2"], x["b2"], R=rows)
        last = rows[torch.tensor([grow[0] - 1, n - 1], device="cuda")].contiguous()
        out = torch.empty((B, d), device="cuda")
        pb.op_layernorm(code, last, G["lnf_g"], G["lnf_b"], out)
        return torch.matmul(out, G["embed"].float().t().contiguous())

    def prompt(l, qkv, q, a):
        for i, (lo, hi) in enumerate(((0, lens[0]), (lens[0], sum(lens)))):
            pb.op_attention(code, qkv[lo:hi], a[lo:hi], 1, hi - lo, H, hd)

    def step(l, qkv, q, a):
        pb.op_paged_attention(code, q, pools[l], state[0], state[1], a.unflatten(1, (H, hd)), workspace=ws)

    seqs = [t[:n].tolist() for t, n in zip(synth.tokens(w), lens)]
    embed = lambda ids, pos: G["embed"].float()[torch.tensor(ids)] + G["pos"].float()[torch.tensor(pos)]  # noqa: E731
    logits = forward(embed(sum(seqs, []), [*range(lens[0]), *range(lens[1])]), lens, prompt)
    alive, scores = torch.ones((B, 1), **i32), torch.zeros((B, 1), device="cuda")
    for k in range(4):
        tokens, parents = torch.empty((B, 1), **i32), torch.empty((B, 1), **i32)
        pb.op_beam_select(logits, scores, alive, scores, tokens, parents, alive, eos=-1, pad=0, workspace=ws)
        for b in range(B):
            one = w.with_(batch=1, seq_len=len(seqs[b]))
            ref, ref_token = oracle.prefill_first_token(one, np.array([seqs[b]], np.int32))
            compare("step %d sequence %d" % (k, b), logits[b:b + 1].cpu().numpy(), [int(tokens[b])], ref, ref_token)
            seqs[b].append(int(tokens[b]))
        if k < 3:
            logits = forward(embed([s[-1] for s in seqs], [len(s) - 1 for s in seqs]), [1, 1], step)
    assert state[1].tolist() == [n + 3 for n in lens]


def test_a_recorded_call_of_many_sequences():
    """One recorded launch of 200 sequences whose lengths change between replays: more pieces and
    fewer, none, and rows past their table."""
    import torch

    from paged_common import dev, make_pool
    from paper_2503_17707_amd import binding as pb

    log("recorded paged attention of many sequences")
    S, ps, pages = 200, 16, 256
    rs = np.random.RandomState(1)
    pool = make_pool(0, "f16", (pages,), 1, ps, 64, "heads")
    tables = dev(np.stack([rs.permutation(pages) for _ in range(S)]).astype(np.int32))
    q = torch.randn((S, 2, 64), generator=torch.Generator().manual_seed(1)).half().cuda()
    lens, out, eager = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.empty_like(q), torch.empty_like(q)
    ws = torch.full((pb.paged_attention_workspace(S, 2, pool, pages),), 255, dtype=torch.uint8, device="cuda")
    run = lambda o: pb.op_paged_attention(1, q, pool, tables, lens, o, scale=0.125, workspace=ws)  # noqa: E731
    run(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out)
    for most in (4096, 30, 4097, 1, 0, 3000, 4096):
        lens.copy_(torch.from_numpy(rs.randint(0, most + 1, S).astype(np.int32)))
        run(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.nan_to_num(7), eager.nan_to_num(7)), most
        assert torch.isnan(out).flatten(1).all(1).tolist() == (lens > 4096).tolist()
        assert torch.all(out[lens == 0] == 0)


def test_the_readme_s_step_runs():
    """The step as the README shows it: scores, parents and alive [prompts, beams], q scaled."""
    import os

    import torch

    from paged_common import attention64, select64
    from paper_2503_17707_amd import binding as pb

    log("the README's step")
    readme = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    code = [b.split("```")[0] for b in readme.split("```python\n")[1:] if "op_page_fork" in b.split("```")[0]]
    assert len(code) == 1
    B, W, L, prompts = 2, 3, 2, (5, 40)
    s = Beams("f16", B, W, L, 4, 2, 64, 16, 50, 60, "rows", 3)
    g = torch.Generator().manual_seed(3)
    s.admit(prompts, [_kv(torch, g, s.dt, sum(prompts), 2, 64) for _ in range(L)])
    s.qkv.copy_(torch.randn(s.qkv.shape, generator=g))
    s.qkv[1] = s.qkv[0]
    s.logits.copy_(torch.randn(s.logits.shape, generator=g))
    s.scores.copy_(-torch.rand(s.scores.shape, generator=g))
    s.alive[1, 2] = 0
    q, k, v = s.split(0)
    want = select64(s.logits.cpu().numpy(), s.scores.cpu().numpy(), s.alive.cpu().numpy(), 2, 1)
    a, b = s.sets
    exec(code[0], dict(pb=pb, dt=s.code, pools=s.pool, parents=s.parents, tables=a["tables"], lens=a["lens"], refs=a["refs"],
                       alive=s.alive, new_tables=b["tables"], start=b["start"], new_lens=b["lens"], new_refs=b["refs"],
                       short=s.short, ws=s.ws, n_layers=L, q=q, k=k, v=v, out=s.out[0], logits=s.logits, scores=s.scores,
                       tokens=s.tokens))
    assert b["lens"].tolist() == [6, 6, 6, 41, 41, 40] and s.short.tolist() == [0, 0]
    ref, tol = attention64(q, s.pool[1], b["tables"].cpu().numpy(), b["lens"].tolist(), 16, 1.0, 0)
    assert torch.all((s.out[0].double().cpu() - ref).abs() <= tol)
    for got, ref in zip((s.tokens, s.parents, s.alive), want[1:]):
        assert np.array_equal(got.cpu().numpy(), ref)


def test_two_streams_at_once():
    """Calls on two streams, each with its own workspace, and a stream passed by argument."""
    import torch

    from paged_common import attention64, dev, make_pool, make_tables
    from paper_2503_17707_amd import binding as pb

    log("paged attention on two streams")
    ps, H, hd, n = 16, 8, 128, 6000
    rs = np.random.RandomState(0)
    tables = make_tables(rs, np.array([n, n]), ps, 2 * (n // ps), n // ps)
    pool = make_pool(0, "bf16", (2 * (n // ps),), 2, ps, hd, "heads")
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    t, lens = [dev(tables[i:i + 1]) for i in range(2)], dev(np.array([n], np.int32))
    qs = [torch.randn((1, H, hd), device="cuda").bfloat16() for _ in range(2)]
    outs = [torch.empty_like(q) for q in qs]
    ws = [torch.empty(pb.paged_attention_workspace(1, H, pool, n // ps), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            pb.op_paged_attention(0, qs[i], pool, t[i], lens, outs[i], scale=0.1, workspace=ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        ref, tol = attention64(qs[i], pool, tables[i:i + 1], [n], ps, 0.1, 0)
        assert torch.all((outs[i].double().cpu() - ref).abs() <= tol)


def test_two_runs_give_the_same_bits():
    import torch

    from paged_common import dev, make_pool, make_tables
    from paper_2503_17707_amd import binding as pb

    log("paged attention twice")
    rs = np.random.RandomState(2)
    lens = np.array([4000, 17, 1500, 0, 2600], np.int32)
    n_pages = int((-(-lens // 16)).sum())
    tables = dev(make_tables(rs, lens, 16, n_pages, 260))
    pool = make_pool(0, "f16", (n_pages,), 4, 16, 64, "rows")
    q = torch.randn((5, 8, 64), device="cuda").half()
    ws = torch.empty(pb.paged_attention_workspace(5, 8, pool, 260), dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(3):
        out = torch.empty_like(q)
        ws.fill_(255)
        pb.op_paged_attention(1, q, pool, tables, dev(lens), out, workspace=ws, shared=len(outs) == 2)
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
