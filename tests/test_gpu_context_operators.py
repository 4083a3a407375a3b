"""Sampled steps, forks and token trees of a context, against the oracle on the same token histories."""
import numpy as np
import pytest
import torch

import operators_plain as plain
from gpu_common import both_models, gpu_context
from helpers import small_cfg
from oracle import oracle as orc
from paper_2509_24007_amd import inputs as syn
from paper_2509_24007_amd import sdlm

pytestmark = pytest.mark.gpu

MODELS = {
    "fp32": (small_cfg(hidden=64, n_q_heads=4, n_kv_heads=2, head_dim=32, ffn=112, vocab=300), 0.3, 1e-4),
    "bf16": (syn.ModelCfg(2, 64, 4, 2, 64, 128, 300, rope_theta=1e4, dtype="bf16"), 0.05, 2e-2),
    "mfma": (syn.ModelCfg(2, 256, 6, 2, 128, 512, 1000, dtype="bf16"), 0.05, 2e-2),
}


def setup(kind, lens, D, *, seed=5, paged=True, n_pages=60, max_batch=6, max_seq_len=200, tau=0.4, **kw):
    m, std, tol = MODELS[kind]
    if kw.pop("causal", False):
        m = m.__class__(**{**m.__dict__, "block_causal": True})
    om, g, layers = both_models(m, seed=seed, std=std)
    ctx = gpu_context(m, g, layers, max_batch=max_batch, max_seq_len=max_seq_len, D=D, tau=tau, paged=paged, n_pages=n_pages if paged else 0, **kw)
    prompts = [syn.uniform_int(seed, f"p{i}", n, 0, m.vocab - 1).numpy() for i, n in enumerate(lens)]
    ctx.prefill(prompts)
    return ctx, om, m, tol, [list(map(int, p)) for p in prompts]


class Step:
    """One decode_step with all of its outputs."""

    def __init__(self, ctx, m):
        B, D = ctx.batch, ctx.D
        self.ids = torch.full((B, D), -7, dtype=torch.int32, device="cuda")
        self.count = torch.full((B,), -7, dtype=torch.int32, device="cuda")
        self.conf = torch.zeros(B, D, device="cuda")
        self.logits = torch.full((B, D, m.vocab), float("nan"), device="cuda")
        ctx.decode_step(self.ids, self.count, self.conf, self.logits)


def check_history(ctx, om, m, tol, history, tau=0.4):
    """The next step of every sequence is that of its token history alone."""
    st = Step(ctx, m)
    n, _ = ctx.get_lengths()
    assert n.tolist() == [len(h) for h in history]
    for b, h in enumerate(history):
        seq = orc.Seq(om, len(h) + 2 * ctx.D)
        seq.prefill(np.array(h))
        z = seq.step(ctx.D, tau)[0]
        err = np.max(np.abs(st.logits[b].cpu().numpy() - z), axis=1) / np.max(np.abs(z), axis=1)
        assert err.max() <= tol, (b, err)
    return st


def commit(ctx, history, ids, counts):
    ctx.kv_commit(torch.tensor(ids, dtype=torch.int32).cuda(), torch.tensor(counts, dtype=torch.int32).cuda())
    for b, (row, c) in enumerate(zip(ids, counts)):
        history[b] += [int(v) for v in row[:c]]


# ---------------------------------------------------------------------------------------------------------------- sampled steps

@pytest.mark.parametrize("kind,conf_fn,rule", [("fp32", 0, 0), ("fp32", 1, 1), ("mfma", 0, 1), ("bf16", 1, 0)])
@pytest.mark.parametrize("D", [1, 4])
def test_sampled_step(kind, conf_fn, rule, D):
    ctx, om, m, tol, hist = setup(kind, [20, 3, 33], D, conf_fn=conf_fn, accept_rule=rule)
    rng = np.random.default_rng(D)
    for step in range(3):
        st = check_history(ctx, om, m, tol, hist)
        if step == 0:      # a second round on the same step: nothing random left at temperature 0
            ids, cnt, conf = torch.zeros_like(st.ids), torch.zeros_like(st.count), torch.zeros_like(st.conf)
            ctx.sample_step(st.logits, torch.rand(3, D, device="cuda"), ids, cnt, conf, temperature=torch.zeros(3, D, device="cuda"))
            torch.cuda.synchronize()
            assert torch.equal(ids, st.ids) and torch.equal(cnt, st.count) and torch.equal(conf, st.conf)
        u, t, k = [torch.from_numpy(v).cuda() for v in (rng.random((3, D), dtype=np.float32), rng.choice([0.5, 1.0, 2.0], (3, D)).astype(np.float32), rng.choice([0, 3, 40], (3, D)).astype(np.int32))]
        ids, cnt, conf = torch.zeros_like(st.ids), torch.zeros_like(st.count), torch.zeros_like(st.conf)
        ctx.sample_step(st.logits, u, ids, cnt, conf, temperature=t, top_k=k)
        torch.cuda.synchronize()
        z = st.logits.double().cpu().numpy()
        for b in range(3):
            for j in range(D):
                assert ids[b, j].item() == plain.sample_row(z[b, j], t[b, j].item(), k[b, j].item(), 1.0, 0.0, u[b, j].item())[0]
                w = np.exp(z[b, j] - z[b, j].max())
                # the step's own confidence is within fp32 sums over the vocabulary (2^-24 sqrt(V) and its exponentials' few 2^-24) of the exact one; then two roundings and an exponential
                want = w[ids[b, j].item()] / w.sum() if conf_fn == 0 else st.conf[b, j].item()
                assert abs(conf[b, j].item() - want) <= 64 * 2.0 ** -24 * want
            assert cnt[b].item() == orc.gamma(conf[b].cpu().numpy(), 0.4, rule)
        ctx.kv_commit()
        for b in range(3):
            hist[b] += ids[b, :cnt[b].item()].tolist()
    check_history(ctx, om, m, tol, hist)
    ctx.close()


def test_sampled_step_refusals_and_masked_rows():
    ctx, om, m, tol, hist = setup("fp32", [5], 4)
    u = torch.rand(1, 4, device="cuda")
    ids, cnt, z = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(4, 300, device="cuda")
    with pytest.raises(sdlm.SdlmError) as e:
        ctx.sample_step(z, u, ids, cnt)
    assert e.value.code == sdlm.ESTATE
    st = Step(ctx, m)
    for bad in (dict(u=u[:, :2]), dict(logits=z[:3]), dict(logits=z.double()), dict(temperature=torch.zeros(4)), dict(top_k=u)):
        kw = dict(logits=z, u=u, ids=ids, count=cnt)
        kw.update(bad)
        with pytest.raises(sdlm.SdlmError) as e:
            ctx.sample_step(kw.pop("logits"), kw.pop("u"), kw.pop("ids"), kw.pop("count"), **kw)
        assert e.value.code == sdlm.EINVAL
    masked = st.logits.clone()
    masked[0, 1] = -float("inf")
    ctx.sample_step(masked, u, ids, cnt, temperature=torch.zeros(1, 4, device="cuda"))
    assert torch.equal(ids, st.ids)      # a position without a token keeps its own
    ctx.close()


def test_sampled_step_of_many_rows():
    """More rows than a launch draws for at once."""
    ctx, om, m, tol, hist = setup("fp32", [3 + i % 5 for i in range(70)], 4, max_batch=70, n_pages=300)
    st = Step(ctx, m)
    u = torch.rand(70, 4, generator=torch.Generator().manual_seed(1)).cuda()
    ids, cnt = torch.zeros_like(st.ids), torch.zeros_like(st.count)
    ctx.sample_step(st.logits, u, ids, cnt)
    want, _ = sdlm.sample(st.logits.view(280, -1), u.view(-1))
    assert torch.equal(ids.view(-1), want)
    ctx.close()


# ---------------------------------------------------------------------------------------------------------------- forks

@pytest.mark.parametrize("kind,paged", [("fp32", True), ("fp32", False), ("mfma", True), ("mfma", False)])
def test_forked_sequences_go_their_own_ways(kind, paged):
    D = 4
    ctx, om, m, tol, hist = setup(kind, [37, 16], D, paged=paged)
    rng = np.random.default_rng(3)

    def some(B):
        return rng.integers(0, m.vocab, (B, D)).tolist(), rng.integers(1, D + 1, B).tolist()

    for parents in ([0, 0, 1, 0], [3, 1, 1, 0, 0, 2], [1, 0], [0, 0, 1, 1, 0, 0], [5], [0, 0]):
        ctx.fork(parents)
        hist = [list(hist[p]) for p in parents]
        for _ in range(2):
            check_history(ctx, om, m, tol, hist)
            commit(ctx, hist, *some(len(parents)))
    check_history(ctx, om, m, tol, hist)
    ctx.close()


@pytest.mark.parametrize("paged", [True, False])
def test_forks_of_a_large_context(paged):
    """64 sequences of up to 8192 tokens: a table of 32768 pages, more than one workgroup plans."""
    D = 4
    ctx, om, m, tol, hist = setup("fp32", [37, 16, 300], D, paged=paged, max_batch=64, max_seq_len=8192, n_pages=120)
    rng = np.random.default_rng(4)
    for parents in ([0, 2, 1, 2, 2], [4, 4, 0, 1], [3, 1, 0, 0, 2, 2, 1]):
        ctx.fork(parents)
        hist = [list(hist[p]) for p in parents]
        check_history(ctx, om, m, tol, hist)
        commit(ctx, hist, rng.integers(0, m.vocab, (len(parents), D)).tolist(), rng.integers(1, D + 1, len(parents)).tolist())
    check_history(ctx, om, m, tol, hist)
    ctx.close()


def test_fork_shares_pages_and_frees_them():
    """Six samples of a prompt of 100 tokens in a pool of 20 pages: unshared they would need 42; then again and again without a leak."""
    ctx, om, m, tol, hist = setup("fp32", [100], 4, n_pages=20)
    for round_ in range(4):
        ctx.fork([0] * 6)
        hist = [list(hist[0]) for _ in range(6)]
        st = Step(ctx, m)
        ids = [[(7 * round_ + b + j) % m.vocab for j in range(4)] for b in range(6)]
        commit(ctx, hist, ids, [2] * 6)
        keep = round_ % 6
        ctx.fork([keep])
        hist = [hist[keep]]
    check_history(ctx, om, m, tol, hist)
    ctx.close()


def test_fork_refusals():
    ctx, om, m, tol, hist = setup("fp32", [60, 30], 4, n_pages=8)      # 4 + 2 pages held
    fresh = sdlm.Context(sdlm.model_cfg(m), max_batch=2, max_seq_len=64, block_D=4, tau=0.5)
    with pytest.raises(sdlm.SdlmError) as e:
        fresh.fork([0])
    assert e.value.code == sdlm.ESTATE
    for parents in ([], [0] * 7, [0, 2], [-1, 0]):
        with pytest.raises(sdlm.SdlmError) as e:
            ctx.fork(parents)
        assert e.value.code == sdlm.EINVAL
    with pytest.raises(sdlm.SdlmError) as e:
        ctx.fork([0, 0, 0, 0, 1, 1])      # four open pages, two free
    assert e.value.code == sdlm.ECAPACITY
    check_history(ctx, om, m, tol, hist)
    ctx.fork([0, 1, 0])                   # one open page
    hist = [hist[0], hist[1], list(hist[0])]
    check_history(ctx, om, m, tol, hist)
    commit(ctx, hist, [[1, 2, 3, 4]] * 3, [1, 4, 1])      # at most 64, 34 and 64 positions: 4 + 3 + 4 pages, three of them shared, and there are 8
    check_history(ctx, om, m, tol, hist)
    with pytest.raises(sdlm.SdlmError) as e:              # now 65, 38 and 65: 5 + 3 + 5 less three
        ctx.kv_commit()
    assert e.value.code == sdlm.ECAPACITY
    ctx.close()
    fresh.close()


# ---------------------------------------------------------------------------------------------------------------- trees

def node_logits(om, history, tokens, parents, i, D):
    branch, j = [], i
    while j >= 0:
        branch.append(int(tokens[j]))
        j = int(parents[j])
    h = list(history) + branch[::-1]
    seq = orc.Seq(om, len(h) + 2 * D)
    seq.prefill(np.array(h))
    return seq.step(D, 0.4)[0][0]


def walk(first, tokens, parents, preds):
    at, y, path = -1, first, []
    for i in range(len(tokens)):
        if parents[i] == at and tokens[i] == y:
            at, y = i, preds[i]
            path.append(i)
    return path, y


def grow(ctx, m, st, B, T, rng):
    """Trees of T nodes in which a branch is right as far as it goes: the model's own predictions, with wrong nodes between them."""
    tokens = rng.integers(0, m.vocab, (B, T)).astype(np.int32)
    parents = np.array([[int(rng.integers(-1, i)) if i else -1 for i in range(T)] for _ in range(B)], np.int32)
    right, y = [-1] * B, st.ids[:, 0].tolist()
    z = torch.zeros(B, T, m.vocab, device="cuda")
    for i in range(0, T, 2):
        for b in range(B):
            if b % 3 != 2 or i == 0:
                tokens[b, i], parents[b, i] = y[b], right[b]
        ctx.verify_tree(torch.from_numpy(tokens).cuda(), torch.from_numpy(parents).cuda(), logits=z)
        pred = z.argmax(2)
        for b in range(B):
            if b % 3 != 2 or i == 0:
                right[b], y[b] = i, pred[b, i].item()
    return tokens, parents


@pytest.mark.parametrize("kind,D,T,paged", [("fp32", 4, 12, True), ("fp32", 4, 1, False), ("fp32", 1, 16, True), ("fp32", 2, 10, False), ("fp32", 8, 14, True), ("fp32", 16, 15, True), ("fp32", 3, 7, False),
                                            ("mfma", 4, 12, True), ("mfma", 1, 16, False), ("mfma", 8, 9, True), ("mfma", 16, 15, False), ("bf16", 4, 12, True), ("bf16", 1, 5, False)])
def test_verified_trees(kind, D, T, paged):
    ctx, om, m, tol, hist = setup(kind, [20, 1, 47, 16], D, paged=paged)
    rng = np.random.default_rng(D * 100 + T)
    B = 4
    for step in range(3):
        st = check_history(ctx, om, m, tol, hist)
        tokens, parents = grow(ctx, m, st, B, T, rng)
        z = torch.full((B, T, m.vocab), float("nan"), device="cuda")
        path, count, nxt = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B, T), (B,), (B,))]
        ctx.verify_tree(torch.from_numpy(tokens).cuda(), torch.from_numpy(parents).cuda(), path, count, nxt, z)
        torch.cuda.synchronize()
        g = z.cpu().numpy()
        for b in range(B):
            for i in range(0, T, 1 if b == 0 else 3):
                ref = node_logits(om, hist[b], tokens[b], parents[b], i, D)
                assert np.max(np.abs(g[b, i] - ref)) / np.max(np.abs(ref)) <= tol, (step, b, i)
            want, y = walk(st.ids[b, 0].item(), tokens[b], parents[b], g[b].argmax(1))
            assert count[b].item() == len(want) and path[b].tolist() == want + [-1] * (T - len(want)) and nxt[b].item() == y
            assert len(want) >= 1
            if step < 2:
                hist[b] += [int(tokens[b, i]) for i in want] + [y]
        if step < 2:
            n0, _ = ctx.get_lengths()
            ctx.tree_commit()
            n, c = ctx.get_lengths()
            assert n.tolist() == [len(h) for h in hist] and c.tolist() == [len(h) - 1 for h in hist]
        else:      # the step's own result can be committed as if there had been no tree
            ids, cnt = st.ids.tolist(), st.count.tolist()
            ctx.kv_commit()
            for b in range(B):
                hist[b] += ids[b][:cnt[b]]
    check_history(ctx, om, m, tol, hist)
    ctx.close()


@pytest.mark.parametrize("hidden", [256, 3200])      # down by split sums; by whole ones, which carry the norm across the layers
@pytest.mark.parametrize("D,T", [(1, 16), (1, 1), (2, 5), (4, 3)])
def test_trees_of_one_bf16_sequence(D, T, hidden, monkeypatch):
    """At most 16 rows: the kernels of few rows, whose sums of squares lie where the attention's partial results do."""
    monkeypatch.setitem(MODELS, "few", (syn.ModelCfg(3, hidden, 6, 2, 128, 512, 1000, dtype="bf16"), 0.05 if hidden < 1000 else 0.02, 2e-2))
    ctx, om, m, tol, hist = setup("few", [600], D, max_batch=1, max_seq_len=700)
    assert T * (D + 1 if D > 1 else 1) <= 16
    rng = np.random.default_rng(D)
    for step in range(2):
        st = check_history(ctx, om, m, tol, hist)
        tokens, parents = grow(ctx, m, st, 1, T, rng)
        z = torch.full((1, T, m.vocab), float("nan"), device="cuda")
        path, count, nxt = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((1, T), (1,), (1,))]
        ctx.verify_tree(torch.from_numpy(tokens).cuda(), torch.from_numpy(parents).cuda(), path, count, nxt, z)
        g = z.cpu().numpy()
        for i in range(T):
            ref = node_logits(om, hist[0], tokens[0], parents[0], i, D)
            assert np.max(np.abs(g[0, i] - ref)) / np.max(np.abs(ref)) <= tol, (step, i)
        want, y = walk(st.ids[0, 0].item(), tokens[0], parents[0], g[0].argmax(1))
        assert len(want) >= 1 and path[0].tolist() == want + [-1] * (T - len(want)) and count.item() == len(want) and nxt.item() == y
        ctx.tree_commit()
        hist[0] += [int(tokens[0, i]) for i in want] + [y]
    check_history(ctx, om, m, tol, hist)
    ctx.close()


@pytest.mark.parametrize("heads,d", [(160, 128), (600, 32)])
def test_trees_of_many_kv_heads(heads, d, monkeypatch):
    """More kv heads than 8 MB of partial results hold, and more rows than the small launch takes."""
    monkeypatch.setitem(MODELS, "wide", (small_cfg(hidden=64, n_q_heads=heads, n_kv_heads=heads, head_dim=d, ffn=112, vocab=300, n_layers=1), 0.1, 1e-4))
    ctx, om, m, tol, hist = setup("wide", [70], 4, max_batch=1)
    st = check_history(ctx, om, m, tol, hist)
    tokens, parents = grow(ctx, m, st, 1, 12, np.random.default_rng(2))
    z = torch.zeros(1, 12, m.vocab, device="cuda")
    ctx.verify_tree(torch.from_numpy(tokens).cuda(), torch.from_numpy(parents).cuda(), logits=z)
    for i in range(0, 12, 3):
        ref = node_logits(om, hist[0], tokens[0], parents[0], i, 4)
        assert np.max(np.abs(z[0, i].cpu().numpy() - ref)) / np.max(np.abs(ref)) <= tol
    ctx.close()


@pytest.mark.parametrize("kind", ["fp32", "mfma"])
def test_trees_of_the_causal_block(kind):
    ctx, om, m, tol, hist = setup(kind, [20, 9, 30], 4, causal=True)
    rng = np.random.default_rng(8)
    st = check_history(ctx, om, m, tol, hist)
    tokens, parents = grow(ctx, m, st, 3, 12, rng)
    z = torch.zeros(3, 12, m.vocab, device="cuda")
    ctx.verify_tree(torch.from_numpy(tokens).cuda(), torch.from_numpy(parents).cuda(), logits=z)
    for b in range(3):
        for i in range(0, 12, 2):
            ref = node_logits(om, hist[b], tokens[b], parents[b], i, 4)
            assert np.max(np.abs(z[b, i].cpu().numpy() - ref)) / np.max(np.abs(ref)) <= tol
    ctx.close()


def test_tree_on_the_cache_is_what_pending_rows_write():
    """K/V that a tree's commit moves into the cache against those that the ordinary way writes there, and the oracle's."""
    ctx, om, m, tol, hist = setup("fp32", [30], 4)
    st = check_history(ctx, om, m, tol, hist)
    tokens, parents = grow(ctx, m, st, 1, 12, np.random.default_rng(1))
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    path = torch.zeros(1, 12, dtype=torch.int32, device="cuda")
    ctx.verify_tree(torch.from_numpy(tokens).cuda(), torch.from_numpy(parents).cuda(), path, count)
    ctx.tree_commit()
    g = count.item()
    assert g >= 5
    seq = orc.Seq(om, 80)
    seq.prefill(np.array(hist[0] + [int(tokens[0, i]) for i in path[0, :g].tolist()]))
    for layer in range(2):
        for h in range(2):
            k, v = ctx.read_kv(layer, 0, h, 0, 30 + g)
            for p in range(30 + g):
                ko, vo = seq.read_kv(layer, p, h)
                assert np.max(np.abs(k[p].numpy() - ko)) <= 1e-4 * max(1.0, np.max(np.abs(ko))) and np.max(np.abs(v[p].numpy() - vo)) <= 1e-4 * max(1.0, np.max(np.abs(vo)))
    ctx.close()


def test_tree_padding_and_bad_nodes():
    ctx, om, m, tol, hist = setup("fp32", [12, 25], 4)
    st = Step(ctx, m)
    good = st.ids[:, 0].tolist()
    path, count = torch.zeros(2, 5, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    # negative tokens are no nodes; sequence 1 has none at all
    tok = torch.tensor([[-1, good[0], -1, 5, -1], [-1] * 5], dtype=torch.int32).cuda()
    par = torch.tensor([[-1, -1, 1, 1, 3], [-1] * 5], dtype=torch.int32).cuda()
    ctx.verify_tree(tok, par, path, count)
    assert count.tolist()[0] >= 1 and path[0, 0].item() == 1 and count.tolist()[1] == 0
    ctx.get_lengths()
    # a parent behind its node, one that does not exist, a token beyond the vocabulary: out, and reported
    tok = torch.tensor([[good[0], good[0], 300, good[0], 7], [good[1], 1, 2, 3, 4]], dtype=torch.int32).cuda()
    par = torch.tensor([[3, -2, -1, -1, 9], [-1, 0, 0, 0, 0]], dtype=torch.int32).cuda()
    ctx.verify_tree(tok, par, path, count)
    assert path[0, 0].item() == 3 and path[1, 0].item() == 0
    with pytest.raises(sdlm.SdlmError) as e:
        ctx.get_lengths()
    assert e.value.code == sdlm.EINVAL
    ctx.tree_commit()
    n, c = ctx.get_lengths()
    assert n.tolist() == [12 + count[0].item() + 1, 25 + count[1].item() + 1]
    ctx.close()


def test_tree_refusals():
    ctx, om, m, tol, hist = setup("fp32", [150, 40], 4, max_seq_len=170, n_pages=14)
    tok, par = torch.zeros(2, 12, dtype=torch.int32, device="cuda"), torch.full((2, 12), -1, dtype=torch.int32, device="cuda")

    def refused(code, f, *a, **k):
        with pytest.raises(sdlm.SdlmError) as e:
            f(*a, **k)
        assert e.value.code == code

    refused(sdlm.ESTATE, ctx.verify_tree, tok, par)
    refused(sdlm.ESTATE, ctx.tree_commit)
    Step(ctx, m)
    refused(sdlm.ESTATE, ctx.tree_commit)
    refused(sdlm.EINVAL, ctx.verify_tree, tok[:, :0], par[:, :0])
    refused(sdlm.EINVAL, ctx.verify_tree, torch.zeros(2, 13, dtype=torch.int32, device="cuda"), torch.zeros(2, 13, dtype=torch.int32, device="cuda"))
    refused(sdlm.EINVAL, ctx.verify_tree, tok, par[:, :3])
    refused(sdlm.EINVAL, ctx.verify_tree, tok.long(), par.long())
    refused(sdlm.EINVAL, ctx.verify_tree, tok, par, count=torch.zeros(1, dtype=torch.int32, device="cuda"))
    ctx.verify_tree(tok, par)             # 150 + 12 + 4 <= 170
    ctx.verify_step(0)                    # takes the same staging tiles
    refused(sdlm.ESTATE, ctx.tree_commit)
    ctx.verify_tree(tok, par)
    refused(sdlm.ECAPACITY, ctx.tree_commit)      # 13 pages held, one free; both sequences may grow by 13 tokens
    ctx.kv_commit(torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.tensor([4, 1], dtype=torch.int32).cuda())
    refused(sdlm.ESTATE, ctx.verify_tree, tok, par)
    Step(ctx, m)
    ctx.verify_tree(tok, par)             # 154 + 12 + 4 <= 170
    ctx.kv_commit(torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.tensor([1, 1], dtype=torch.int32).cuda())
    Step(ctx, m)
    refused(sdlm.ECAPACITY, ctx.verify_tree, tok, par)     # 155 + 12 + 4
    ctx.verify_tree(tok[:, :11].contiguous(), par[:, :11].contiguous())
    ctx.close()


def test_samples_forks_and_trees_together():
    """A search as a program runs it: one prompt, four samples, drafts verified as trees, the two best go on, sampled tokens between."""
    D = 4
    ctx, om, m, tol, hist = setup("fp32", [33], D, n_pages=40)
    rng = np.random.default_rng(0)
    ctx.fork([0] * 4)
    hist = [list(hist[0]) for _ in range(4)]
    for step in range(4):
        st = check_history(ctx, om, m, tol, hist)
        B = len(hist)
        if step % 2 == 0:
            ids, cnt = torch.zeros_like(st.ids), torch.zeros_like(st.count)
            ctx.sample_step(st.logits, torch.from_numpy(rng.random((B, D), dtype=np.float32)).cuda(), ids, cnt)
            ctx.kv_commit()
            for b in range(B):
                hist[b] += ids[b, :cnt[b].item()].tolist()
        else:
            tokens, parents = grow(ctx, m, st, B, 8, rng)
            path, count, nxt = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((B, 8), (B,), (B,))]
            ctx.verify_tree(torch.from_numpy(tokens).cuda(), torch.from_numpy(parents).cuda(), path, count, nxt)
            ctx.tree_commit()
            for b in range(B):
                hist[b] += [int(tokens[b, i]) for i in path[b, :count[b].item()].tolist()] + [nxt[b].item()]
            keep = [3, 1, 1, 3, 0]
            ctx.fork(keep)
            hist = [list(hist[k]) for k in keep]
    check_history(ctx, om, m, tol, hist)
    ctx.close()


def test_captured_samples_and_trees():
    """A sampled step with its commit and a verified tree with its own, each in a caller's graph, replayed in turn: an eager context on the same inputs draws, accepts and publishes the same."""
    D, T, B = 4, 6, 2
    side = torch.cuda.Stream()
    eager, om, m, tol, _ = setup("fp32", [33, 18], D)
    replayed = setup("fp32", [33, 18], D, stream=side)[0]
    i32 = dict(dtype=torch.int32, device="cuda")
    u = torch.zeros(B, D, device="cuda")
    tokens, parents = torch.zeros(B, T, **i32), torch.zeros(B, T, **i32)
    outs = []
    for _ in range(2):
        outs.append(dict(ids=torch.zeros(B, D, **i32), count=torch.zeros(B, **i32), z=torch.zeros(B, D, m.vocab, device="cuda"), drawn=torch.zeros(B, D, **i32), n=torch.zeros(B, **i32),
                         path=torch.zeros(B, T, **i32), g=torch.zeros(B, **i32), next=torch.zeros(B, **i32)))
    torch.cuda.synchronize()

    def sampled(ctx, o):
        ctx.decode_step(o["ids"], o["count"], None, o["z"])
        ctx.sample_step(o["z"], u, o["drawn"], o["n"])
        ctx.kv_commit()

    def tree(ctx, o):
        ctx.decode_step(o["ids"], o["count"], None, o["z"])
        ctx.verify_tree(tokens, parents, o["path"], o["g"], o["next"])
        ctx.tree_commit()

    graphs = []
    for f in (sampled, tree):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side, capture_error_mode="thread_local"):
            f(replayed, outs[1])
        graphs.append(graph)
    rng = np.random.default_rng(3)
    accepted = 0
    for step in range(6):
        u.copy_(torch.from_numpy(rng.random((B, D), dtype=np.float32)))
        f = (sampled, tree)[step % 2]
        if f is tree:
            st = Step(eager, m)
            tk, pr = grow(eager, m, st, B, T, rng)
            tokens.copy_(torch.from_numpy(tk))
            parents.copy_(torch.from_numpy(pr))
        torch.cuda.synchronize()
        f(eager, outs[0])
        graphs[step % 2].replay()
        torch.cuda.synchronize()
        names = ("ids", "drawn", "n") if f is sampled else ("ids", "path", "g", "next")
        for name in names:
            assert torch.equal(outs[0][name], outs[1][name]), (step, name)
        accepted += int(outs[0]["g"].sum()) if f is tree else 0
        assert eager.get_lengths()[0].tolist() == replayed.get_lengths()[0].tolist()
    assert accepted > 0
    eager.close()
    replayed.close()


def test_tree_behind_a_callers_graph_that_fills_the_context():
    """A caller's graph commits until no position is left, which the host does not see: a tree behind it is computed (its positions end with the rotation's) and cannot be published."""
    D = 4
    side = torch.cuda.Stream()
    ctx, om, m, tol, hist = setup("fp32", [20], D, max_batch=1, max_seq_len=64, stream=side)
    ovr, full = torch.ones(1, D, dtype=torch.int32, device="cuda"), torch.full((1,), D, dtype=torch.int32, device="cuda")
    ids, cnt = torch.zeros_like(ovr), torch.zeros_like(full)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side, capture_error_mode="thread_local"):
        ctx.decode_step(ids, cnt)
        ctx.kv_commit(ovr, full)
    for _ in range(11):
        graph.replay()
    torch.cuda.synchronize()
    z = torch.zeros(1, 12, m.vocab, device="cuda")
    chain = torch.arange(-1, 11, dtype=torch.int32, device="cuda")[None].contiguous()
    ctx.decode_step(ids, cnt)
    ctx.verify_tree(torch.ones(1, 12, dtype=torch.int32, device="cuda"), chain, logits=z)
    ctx.tree_commit()
    torch.cuda.synchronize()
    assert torch.isfinite(z).all()
    with pytest.raises(sdlm.SdlmError) as e:
        ctx.get_lengths()
    assert e.value.code == sdlm.ECAPACITY
    ctx.close()


def test_described_cache_is_not_forked():
    """Pages are handed out by the context's own calls: the fork on the caller's tensors refuses them, before and behind a commit that takes some."""
    import ctypes as C
    ctx, om, m, tol, hist = setup("fp32", [16, 7], 4)
    for _ in range(2):
        desc = sdlm.KvDesc()
        assert ctx.L.sdlm_kv_describe(ctx.h, C.byref(desc)) == 0
        assert desc.n_pages == 0 and not (desc.backed or desc.page_refs or desc.free_pages or desc.free_count)
        assert ctx.L.sdlm_kv_fork_workspace_bytes(C.byref(desc)) == 0
        some = torch.zeros(1 << 20, dtype=torch.int32, device="cuda")
        assert ctx.L.sdlm_kv_fork(C.byref(desc), some.data_ptr(), 2, 1, some.data_ptr(), some.data_ptr(), 4 << 20, None) == sdlm.EINVAL
        assert "n_pages" in ctx.L.sdlm_op_error().decode()
        check_history(ctx, om, m, tol, hist)
        commit(ctx, hist, [[1, 2, 3, 4]] * 2, [2, 1])
    ctx.fork([1, 0, 1])
    hist = [list(hist[p]) for p in (1, 0, 1)]
    check_history(ctx, om, m, tol, hist)
    ctx.close()


def test_described_cache_serves_the_operators():
    """Attention over a context's own cache through sdlm_kv_describe: a node that sees only the cache is a query over it."""
    import ctypes as C
    ctx, om, m, tol, hist = setup("fp32", [40, 7], 4)
    desc = sdlm.KvDesc()
    assert ctx.L.sdlm_kv_describe(ctx.h, C.byref(desc)) == 0
    assert (desc.n_layers, desc.n_kv_heads, desc.head_dim, desc.dtype, desc.max_seqs) == (2, 2, 32, 0, 6)
    q, out = torch.randn(2, 4, 32, device="cuda"), torch.zeros(2, 4, 32, device="cuda")
    offs, mask, tab = torch.tensor([0, 1, 2], dtype=torch.int32).cuda(), torch.zeros(2, 1, dtype=torch.int64).cuda(), torch.zeros(2, 1, dtype=torch.int32).cuda()
    need = ctx.L.sdlm_tree_attention_workspace_bytes(C.byref(desc), 4, 2, 1, 0)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    a = sdlm.TreeArgs(q.data_ptr(), out.data_ptr(), 128, 128, 2, 2, 4, 1, 0, offs.data_ptr(), mask.data_ptr(), 1, 1, tab.data_ptr(), None)
    assert ctx.L.sdlm_tree_attention(C.byref(desc), 1, C.byref(a), ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    for b, n in enumerate((40, 7)):
        for h in range(4):
            k, v = ctx.read_kv(1, b, h // 2, 0, n)
            s = k.double().numpy() @ q[b, h].double().cpu().numpy() / np.sqrt(32)
            w = np.exp(s - s.max())
            assert np.max(np.abs(out[b, h].cpu().numpy() - (w / w.sum()) @ v.double().numpy())) <= 128 * 2.0 ** -24 * np.max(np.abs(v.numpy()))
    ctx.close()
