"""The model behind a shared prefix: ftts_prefill_shared, ftts_decode_step_shared and the scheduler's
shared_prefix, against the oracle's full forward over prefix, own rows and tokens together.  Bars as in
tests/helpers.py (fp32 1e-4 normwise, bf16 storage 3e-2 absolute on logits)."""
import numpy as np
import pytest

from oracle import gpt as ogpt
from paper_2607_21042_amd import ftts, workload
from tests import helpers

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
SHAPE = workload.ModelShape(n_layer=2, d_model=256, n_head=4, d_head=64, d_ff=512, vocab=640)
MODES = {"f32": ftts.F32, "bf16": ftts.BF16, "w8a16": ftts.W8A16, "w4a16": ftts.W4A16}


def weights(mode):
    master = workload.master_weights(SHAPE, seed=3)
    return master if mode == "f32" else workload.bf16_weights(master) if mode == "bf16" else workload.quantisable_weights(master)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Run:
    """A prefix of P rows prefilled once, B sequences of lens[b] own rows (0: none) behind it."""

    def __init__(self, dm, mode, P, lens, steps, seed=5):
        self.dm, self.P, self.lens = dm, P, lens
        B, adt = len(lens), ftts.act_dtype(MODES[mode])
        self.pre = workload.prefix_embeddings([max(P, 1)], SHAPE.d_model, seed=seed, bf16=mode != "f32")[:P]
        self.rows = np.split(workload.prefix_embeddings([max(n, 1) for n in lens], SHAPE.d_model, seed=seed + 1, bf16=mode != "f32"),
                             np.cumsum([max(n, 1) for n in lens])[:-1])
        self.rows = [r[:n] for r, n in zip(self.rows, lens)]
        n_pre = -(-P // 64)
        bt, n_own = helpers.make_block_table([n + steps for n in lens], seed=seed)
        self.kv = ftts.KVCache(SHAPE, MODES[mode], n_own + n_pre, fill=float("nan"))
        self.pages = i32(list(range(n_own, n_own + n_pre)))
        self.pt = ftts.PageTableView(torch.from_numpy(bt).cuda(), i32([0] * B))
        self.ws = torch.zeros(ftts.shared_workspace_bytes(dm.cfg, B, max(sum(lens), P, 1), P, bt.shape[1]), dtype=torch.uint8,
                              device="cuda")
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(adt)  # noqa: E731
        if P:
            ftts.prefill(dm, up(self.pre), [P], ftts.PageTableView(self.pages[None], i32([0])), self.kv, None, self.ws)
        self.prefix = ftts.SharedPrefix(self.pages, P)
        self.last = torch.full((B, SHAPE.vocab), float("nan"), device="cuda")
        some = [b for b in range(B) if lens[b]]
        if some:
            pt = ftts.PageTableView(self.pt.block_table[some], i32([0] * len(some)))
            last = torch.empty((len(some), SHAPE.vocab), device="cuda")
            ftts.prefill_shared(dm, self.prefix, up(np.concatenate([self.rows[b] for b in some])), [lens[b] for b in some], None,
                                [0] * len(some), 0, 0, pt, self.kv, last, self.ws)
            self.last[some] = last
        self.pt.seq_lens.copy_(i32(lens))

    def step(self, tokens, t, hidden=None):
        B = len(self.lens)
        logits, out = torch.empty((B, SHAPE.vocab), device="cuda"), i32([0] * B)
        ftts.decode_step_shared(self.dm, self.prefix, i32(tokens), i32([t] * B), self.pt, self.kv, logits, out, None,
                                ftts.Sampling(1.0, 1, 1.0), self.ws, hidden_out=hidden)
        self.pt.seq_lens.add_(1)
        torch.cuda.synchronize()
        return logits.cpu().numpy(), out.cpu().numpy()


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("P,lens", [(70, [1]), (64, [33, 0]), (1, [5, 64, 65, 0, 130, 2]), (200, [40, 0, 1]), (0, [3, 70]),
                                    (333, [7 + 5 * i % 90 for i in range(33)])])
def test_parity(mode, P, lens):
    inputs = weights(mode)
    dm = ftts.DeviceModel(inputs, SHAPE, MODES[mode])
    om = ogpt.GPT(helpers.oracle_weights(inputs, mode), SHAPE.n_head, SHAPE.d_head)
    T = 3
    fed = workload.random_tokens(T, len(lens), SHAPE.vocab, seed=7)
    print(f"shared prefix: {mode} P {P}, {len(lens)} sequences", flush=True)
    r = Run(dm, mode, P, lens, T)
    hid = torch.empty((len(lens), SHAPE.d_model), device="cuda")
    got = [r.step(fed[t], t, hid if t == T - 1 else None) for t in range(T)]
    for b in sorted({0, 1, 2, 3, 4, 5, len(lens) - 1} & set(range(len(lens)))):
        last, dec, ref_hid = helpers.oracle_teacher_forced(om, np.concatenate([r.pre, r.rows[b]]), fed[:, b], with_hidden=True)
        if lens[b]:
            ok, err = helpers.tolerance_ok(r.last[b].cpu().numpy(), last, mode)
            assert ok, ("prefill", b, err)
        for t in range(T):
            ok, err = helpers.tolerance_ok(got[t][0][b], dec[t], mode)
            assert ok, (b, t, err)
            assert helpers.argmax_agrees(got[t][1][b], dec[t], mode)[0], (b, t)
        ok, err = helpers.tolerance_ok(hid[b].cpu().numpy(), ref_hid[T - 1], mode)
        assert ok, ("hidden", b, err)


def test_prefill_from_text_ids():
    """Conditioning rows shared, text ids each: what ftts_prefill_ids gives for both together."""
    n_text = 50
    master = workload.master_weights(SHAPE, seed=3)
    rng = np.random.default_rng(2)
    master["tok_emb"] = np.concatenate([master["tok_emb"], (rng.standard_normal((n_text, SHAPE.d_model)) * 0.02).astype(np.float32)])
    dm = ftts.DeviceModel(master, SHAPE, ftts.F32)
    P, texts = 34, [9, 1, 40]
    ids = rng.integers(0, n_text, sum(texts)).astype(np.int32)
    cond = workload.prefix_embeddings([P], SHAPE.d_model, seed=4, bf16=False)
    up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    logits = []
    for shared in (True, False):
        kv = ftts.KVCache(SHAPE, ftts.F32, 8)
        ws = torch.zeros(ftts.shared_workspace_bytes(dm.cfg, 3, 200, P, 2), dtype=torch.uint8, device="cuda")
        pt = ftts.PageTableView(i32([[0, 1], [2, 3], [4, 5]]), i32([0] * 3))
        out = torch.empty((3, SHAPE.vocab), device="cuda")
        if shared:
            ftts.prefill(dm, up(cond), [P], ftts.PageTableView(i32([[7]]), i32([0])), kv, None, ws)
            ftts.prefill_shared(dm, ftts.SharedPrefix(i32([7]), P), None, [0] * 3, up(ids), texts, n_text, 0, pt, kv, out, ws)
        else:
            ftts.prefill_ids(dm, up(np.concatenate([cond] * 3)), [P] * 3, up(ids), texts, n_text, 0, pt, kv, out, ws)
        torch.cuda.synchronize()
        logits.append(out.cpu().numpy())
    assert np.abs(logits[0] - logits[1]).max() <= helpers.FP32_REL_TOL * np.abs(logits[1]).max()


@pytest.mark.parametrize("mode,B", [("bf16", 2), ("bf16", 6), ("w4a16", 3)])
def test_steps_captured_with_their_bookkeeping(mode, B):
    """Steps and ftts_advance replayed from a graph give the eager loop's ids and cache, also after a second run on
    the same workspace; a retired slot (token -1) touches nothing."""
    dm = ftts.DeviceModel(weights(mode), SHAPE, MODES[mode])
    greedy, n = ftts.Sampling(1.0, 1, 1.0), 4

    def loop(graph):
        r = Run(dm, mode, 90, [10 + 60 * b for b in range(B)], 2 * n)
        tok, pos, out = i32([SHAPE.start_token] * (B - 1) + [-1]), i32([0] * B), i32([0] * B)
        hist, count, logits = i32([[-1] * B] * 2 * n), i32([0]), torch.empty((B, SHAPE.vocab), device="cuda")

        def steps():
            for _ in range(n):
                ftts.decode_step_shared(dm, r.prefix, tok, pos, r.pt, r.kv, logits, out, None, greedy, r.ws)
                ftts.advance(tok, pos, r.pt.seq_lens, out, None, SHAPE.stop_token, hist, count)
        torch.cuda.synchronize()
        if graph:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                steps()
        for _ in range(2):
            g.replay() if graph else steps()
            torch.cuda.synchronize()
        return hist.cpu(), r.kv.pool.clone(), r.pt.seq_lens.cpu()

    print(f"shared prefix in a graph: {mode} B {B}", flush=True)
    eager, captured = loop(False), loop(True)
    assert torch.equal(eager[0], captured[0]) and torch.equal(eager[2], captured[2])
    assert torch.equal(torch.nan_to_num(eager[1].float()), torch.nan_to_num(captured[1].float()))
    assert (eager[0][:, -1] == -1).all() and (eager[0][:, :-1] >= 0).all()
    assert eager[2][-1] == 10 + 60 * (B - 1) and eager[2][0] == 10 + 2 * n


@pytest.mark.parametrize("mode,slots,graphs", [("f32", 3, False), ("bf16", 3, True), ("bf16", 9, True)])
def test_scheduler_with_a_shared_prefix(mode, slots, graphs):
    from paper_2607_21042_amd import serve
    inputs = weights(mode)
    dm = ftts.DeviceModel(inputs, SHAPE, MODES[mode])
    om = ogpt.GPT(helpers.oracle_weights(inputs, mode), SHAPE.n_head, SHAPE.d_head, dtype=np.float32)
    P, lens = 150, [40, 1, 70, 129, 5, 33, 64, 17, 90, 2, 48]
    budgets = [10, 25, 7, 12, 30, 3, 9, 14, 5, 21, 6]
    flat = workload.prefix_embeddings([P] + lens, SHAPE.d_model, seed=1, bf16=mode != "f32")
    voice, *own = np.split(flat, np.cumsum([P] + lens)[:-1])
    n_pages = 3 * slots + 4 + 3
    sch = serve.Scheduler(dm, SHAPE, max_slots=slots, n_pages=n_pages, max_ctx=max(lens) + max(budgets),
                          sampling=ftts.Sampling(1.0, 1, 1.0), chunk=4, graphs=graphs, shared_prefix=voice)
    assert len(sch.pool.free) == n_pages - 3
    reqs = [sch.submit(serve.Request(prefix=p, max_new=n)) for p, n in zip(own, budgets)]
    print(f"serve behind a shared prefix: {mode} slots={slots} graphs={graphs}", flush=True)
    sch.run()
    assert not sch.busy() and len(sch.pool.free) == n_pages - 3
    for r, p in zip(reqs, own):
        assert r.done and len(r.tokens) == r.max_new and r.tokens[-1] == SHAPE.stop_token
        fed = np.array([SHAPE.start_token] + r.tokens[:-1], dtype=np.int32)
        _, ref = helpers.oracle_teacher_forced(om, np.concatenate([voice, p]), fed)
        for j in range(r.max_new - 1):
            assert helpers.argmax_agrees(r.tokens[j], ref[j], mode)[0], (r.rid, j)
