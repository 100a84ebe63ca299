"""The operators between an actor's products captured in HIP graphs, on several streams, and as two
calls at once: the same bits as alone.

A captured call allocates nothing, records no memset and keeps nothing on the host, so a replay on new
inputs equals the eager call on them."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


class Update:
    """Heads, log-probabilities, both losses and the way back, on buffers of its own."""

    def __init__(self, hl, tokens=600, vocab=5003, responses=30, seed=0, workspace=None):
        self.hl, self.tokens, self.responses, self.seed = hl, tokens, responses, seed
        cuda = dict(device="cuda")
        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        self.rows, self.grads, self.drows = (torch.empty(tokens, 6 * 64, **bf16) for _ in range(3))
        self.w = torch.ones(64, **bf16)
        self.q, self.k = torch.empty(tokens, 4, 64, **bf16), torch.empty(tokens, 2, 64, **bf16)
        self.logits, self.dlogits = (torch.empty(tokens, vocab, **bf16) for _ in range(2))
        self.targets = torch.zeros(tokens, dtype=torch.int64, **cuda)
        self.f = {k: torch.zeros(tokens, **cuda) for k in ("logp", "entropy", "row_max", "log_sum", "old", "ref", "dlogp", "dentropy", "dpref")}
        self.adv, self.dw = torch.zeros(responses, **cuda), torch.zeros(2, 64, **cuda)
        self.offsets = torch.zeros(responses + 1, dtype=torch.int64, **cuda)
        self.mask = torch.zeros(tokens, dtype=torch.uint8, **cuda)
        self.stats, self.pstats = torch.zeros(8, **cuda), torch.zeros(6, **cuda)
        freq = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).float().cuda()
        self.fill(seed)
        angles = dict(inv_freq=freq, w_q=self.w, w_k=self.w)
        f = self.f
        self.descs = [
            hl.qk_norm_rope_desc(q=self.rows[:, :256], k=self.rows[:, 256:], q_out=self.q, k_out=self.k, **angles),
            hl.qk_norm_rope_bwd_desc(dq=self.grads[:, :256].unflatten(1, (4, 64)), dk=self.grads[:, 256:].unflatten(1, (2, 64)),
                                     dq_in=self.drows[:, :256], dk_in=self.drows[:, 256:], q=hl.unit_desc(x=self.rows[:, :256]),
                                     k=hl.unit_desc(x=self.rows[:, 256:]), dw_q=self.dw[0], dw_k=self.dw[1], **angles),
            hl.token_logprobs_desc(self.logits, self.targets, f["logp"], f["entropy"], f["row_max"], f["log_sum"]),
            hl.policy_loss_desc(f["logp"], f["old"], self.adv, logp_ref=f["ref"], entropy=f["entropy"], mask=self.mask, offsets=self.offsets,
                                beta=0.1, entropy_weight=0.01, kl=3, ratio="sequence", mean="sequences", dlogp=f["dlogp"],
                                dentropy=f["dentropy"], stats=self.stats),
            hl.preference_loss_desc(f["logp"], f["ref"], mask=self.mask, offsets=self.offsets, dlogp=f["dpref"], stats=self.pstats),
            hl.token_logprobs_bwd_desc(self.logits, self.targets, f["row_max"], f["log_sum"], f["dlogp"], self.dlogits,
                                       entropy=f["entropy"], dentropy=f["dentropy"])]
        self.need = max(hl.hilore_qk_norm_rope_bwd_workspace_bytes(self.descs[1]), hl.hilore_token_logprobs_workspace_bytes(self.descs[2]),
                        hl.hilore_policy_loss_workspace_bytes(self.descs[3]), hl.hilore_preference_loss_workspace_bytes(self.descs[4]))
        self.ws = torch.empty(self.need, dtype=torch.uint8, **cuda) if workspace is None else workspace

    def fill(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (self.rows, self.grads, self.logits, self.adv):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        self.targets.copy_(torch.randint(-2000, self.logits.shape[1], (self.tokens,), generator=g, device="cuda"))
        for k in ("old", "ref"):
            self.f[k].copy_(-8.0 - torch.rand(self.tokens, generator=g, device="cuda"))
        self.mask.copy_(self.targets >= 0)
        cuts = torch.sort(torch.randint(0, self.tokens + 1, (self.responses - 1,), generator=g, device="cuda")).values
        self.offsets[1:-1] = cuts
        self.offsets[-1] = self.tokens

    def run(self, stream=None, own_workspace=True):
        hl, d, ws = self.hl, self.descs, self.ws if own_workspace else None
        hl.hilore_qk_norm_rope(d[0], stream=stream)
        hl.hilore_qk_norm_rope_bwd(d[1], workspace=ws, stream=stream)
        hl.hilore_token_logprobs(d[2], workspace=ws, stream=stream)
        hl.hilore_policy_loss(d[3], workspace=ws, stream=stream)
        hl.hilore_preference_loss(d[4], workspace=ws, stream=stream)
        hl.hilore_token_logprobs_bwd(d[5], stream=stream)

    def outputs(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.q, self.k, self.drows, self.dw, self.dlogits, self.stats, self.pstats, *self.f.values())]


def same(a, b):
    return [torch.equal(x, y) for x, y in zip(a, b)]


@pytest.mark.parametrize("tokens,vocab", [(600, 5003), (300, 100000), (1500, 40000), (12000, 700)])
@pytest.mark.parametrize("own_workspace", [True, False])
def test_graph_replays(hl, tokens, vocab, own_workspace):
    u = Update(hl, tokens, vocab)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        u.run(own_workspace=own_workspace)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        u.run(own_workspace=own_workspace)
    for seed in (5, 6, 7):
        u.fill(seed)
        u.run()
        eager = u.outputs()
        for t in (u.q, u.k, u.drows, u.dlogits, u.dw, *[u.f[k] for k in ("logp", "dlogp", "dentropy", "dpref")]):
            t.zero_()
        torch.randn(1000, 1000, device="cuda").sum()  # the program's own work in between
        graph.replay()
        assert all(same(u.outputs(), eager))


def test_two_graphs_share_a_workspace(hl):
    """Replayed one after the other: each leaves nothing for the other to read."""
    a = Update(hl, 12000, 700, seed=1)
    b = Update(hl, 400, 90001, seed=2, workspace=torch.empty(0))
    shared = torch.full((max(a.need, b.need),), 0xFF, dtype=torch.uint8, device="cuda")
    a.ws = b.ws = shared
    graphs = []
    for u in (a, b):
        u.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            u.run()
        graphs.append(graph)
    want = []
    for u in (a, b):
        u.run()
        want.append(u.outputs())
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        assert all(same(a.outputs(), want[0])) and all(same(b.outputs(), want[1]))
        shared.fill_(0xFF)


def test_two_threads_two_streams(hl):
    jobs = [Update(hl, 3000, 9001, seed=11), Update(hl, 200, 120001, seed=12)]
    want = []
    for u in jobs:
        u.run()
        want.append(u.outputs())
    streams, errors = [torch.cuda.Stream() for _ in jobs], []

    def work(u, stream):
        try:
            for _ in range(10):
                u.run(stream.cuda_stream)
            stream.synchronize()
        except Exception as e:  # shown below
            errors.append(e)

    threads = [threading.Thread(target=work, args=a) for a in zip(jobs, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for u, w in zip(jobs, want):
        assert all(same(u.outputs(), w))


def test_an_explicit_stream_needs_a_workspace(hl):
    u = Update(hl)
    stream = torch.cuda.Stream()
    for call in (lambda: hl.hilore_policy_loss(u.descs[3], stream=stream.cuda_stream),
                 lambda: hl.hilore_preference_loss(u.descs[4], stream=stream.cuda_stream)):
        with pytest.raises(ValueError, match="workspace"):
            call()
    hl.hilore_token_logprobs(u.descs[2], stream=stream.cuda_stream)  # one segment a row: none is needed
    stream.synchronize()


def test_a_torch_stream_is_followed(hl):
    """Calls under torch.cuda.stream run on it, with a workspace of its own."""
    u = Update(hl, 450, 80001)
    u.run()
    want = u.outputs()
    u.q.zero_(), u.dlogits.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        u.run(own_workspace=False)
    torch.cuda.current_stream().wait_stream(side)
    assert all(same(u.outputs(), want))
