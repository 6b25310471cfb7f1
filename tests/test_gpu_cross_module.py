"""The operators around an attention to states of another length together, as a
module's training step runs them: heads normalised and rotated, a learned
relative position bias between residues and states, the attention, and the
backward of all of it, eager and captured.

Tolerances: 2e-2 normwise per tensor, as for the attention module step (bf16
hand-offs between the operators); the bias table's gradient sums n entries of
dbias, so an error of norm e in it moves an entry by at most sqrt(n) e
(Cauchy-Schwarz): 2e-2 sqrt(n) |dbias of the head|, and in the weights'
gradients 2e-2 of the root of the terms' squares likewise.
"""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from oracle import relpos_oracle as rl
from oracle import rope_oracle as ro
from paper_2404_11068_amd import cross
from paper_2404_11068_amd import graph as gr
from paper_2404_11068_amd import relpos as rp
from paper_2404_11068_amd import rope
from paper_2404_11068_amd import workloads as W
from tests.parity_util import to_f64

pytestmark = pytest.mark.gpu


def _bf(x):
    return W.as_float64(W._store(np.asarray(x, dtype=np.float64), "bf16"), "bf16")


class _Step:
    """Static buffers; q, k, v, gate are views of packed projections."""

    def __init__(self, N=3, Lq=40, Lk=70, H=4, Hk=2, d=32, rot=24, seed=0):
        g = torch.Generator(device="cpu").manual_seed(seed)
        bf = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
        self.shape = (N, Lq, Lk, H, Hk, d)
        self.qg, self.kv = bf(N, Lq, 2 * H, d), bf(N, Lk, 2 * Hk, d)
        self.q, self.gate, self.k, self.v = self.qg[:, :, :H], self.qg[:, :, H:], self.kv[:, :, :Hk], self.kv[:, :, Hk:]
        self.dout = bf(N, Lq, H, d)
        self.mask = (torch.rand(N, Lk, generator=g) < 0.8).to(torch.uint8).cuda()
        self.mask[:, 0] = 1
        self.pos_q = (torch.arange(Lq) * 2 + 5).int().cuda()
        self.pos_k = torch.arange(Lk).int().cuda()
        self.freq = rope.rope_frequencies(rot, 1000.0)
        self.steps = rope.rope_steps(self.freq)
        self.wq, self.wk = (1 + 0.2 * torch.randn(d, generator=g)).cuda(), (1 + 0.2 * torch.randn(d, generator=g)).cuda()
        self.edges = rp.relpos_edges_clip(16)
        self.table = (0.3 * torch.randn(H, self.edges.numel() + 1, generator=g)).cuda()
        self.rq, self.rk, self.rv = torch.empty_like(self.dout), bf(N, Lk, Hk, d), None
        self.bias = torch.empty(1, H, Lq, Lk, dtype=torch.bfloat16, device="cuda")
        self.dbias, self.dbias32 = torch.empty_like(self.bias), torch.empty(1, H, Lq, Lk, device="cuda")
        self.out, self.lse = torch.empty_like(self.dout), torch.empty(N, H, Lq, device="cuda")
        self.dqg, self.dkv = torch.empty_like(self.qg), torch.empty_like(self.kv)
        # gradients at the rotated heads; those of v and gate go straight into the packed ones
        self.gq, self.gg, self.gk, self.gv = (torch.empty_like(t) for t in (self.rq, self.rq, self.rk, self.rk))
        self.dwq, self.dwk, self.dtable = torch.empty_like(self.wq), torch.empty_like(self.wk), torch.empty_like(self.table)
        self.vc, self.gc = torch.empty_like(self.rk), torch.empty_like(self.rq)
        self.ws_f = torch.empty(max(cross.cross_attn_fwd_workspace_size(self.rq, self.rk), 1), dtype=torch.uint8, device="cuda")
        self.ws_b = torch.empty(cross.cross_attn_bwd_workspace_size(self.rq, self.rk, True, True), dtype=torch.uint8, device="cuda")
        self.ws_r = torch.empty(rope.rope_bwd_workspace_size(self.q, self.steps, k=self.k, norm=True), dtype=torch.uint8, device="cuda")
        self.ws_p = torch.empty(max(rp.relpos_bias_bwd_workspace_size(1, H, Lq, Lk, self.edges.numel()), 16), dtype=torch.uint8,
                                device="cuda")

    def first(self, s):
        norm = dict(norm=True, weight_q=self.wq, weight_k=self.wk, stream=s)
        rope.rope_fwd(self.q, self.pos_q, self.steps, k=self.k, pos_k=self.pos_k, out_q=self.rq, out_k=self.rk, **norm)
        # the gate has the rotated queries' layout, the values the rotated keys': rotations by nothing copy them
        none = self.steps[:0]
        rope.rope_fwd(self.gate, self.pos_q, none, k=self.v, pos_k=self.pos_k, out_q=self.gc, out_k=self.vc, stream=s)
        rp.relpos_bias_fwd(self.pos_q.view(1, -1), self.pos_k.view(1, -1), self.edges, self.table, out=self.bias, stream=s)
        cross.cross_attn_fwd(self.rq, self.rk, self.vc, self.gc, self.bias, self.mask, out=self.out, lse=self.lse,
                             workspace=self.ws_f, stream=s)
        cross.cross_attn_bwd(self.rq, self.rk, self.vc, self.gc, self.bias, self.mask, self.out, self.lse, self.dout,
                             dq=self.gq, dk=self.gk, dv=self.gv, dgate=self.gg, dbias=self.dbias, workspace=self.ws_b, stream=s)
        H, Hk = self.shape[3:5]
        rope.rope_bwd(self.gq, self.pos_q, self.steps, dk=self.gk, pos_k=self.pos_k, q=self.q, k=self.k,
                      out_q=self.dqg[:, :, :H], out_k=self.dkv[:, :, :Hk], dweight_q=self.dwq, dweight_k=self.dwk,
                      workspace=self.ws_r, **norm)

    def second(self, s):
        rp.relpos_bias_bwd(self.pos_q.view(1, -1), self.pos_k.view(1, -1), self.edges, self.dbias32, dtable=self.dtable,
                           workspace=self.ws_p, stream=s)

    def outputs(self):
        H, Hk = self.shape[3:5]
        return dict(rq=self.rq, rk=self.rk, bias=self.bias, out=self.out, lse=self.lse, dq=self.dqg[:, :, :H],
                    dk=self.dkv[:, :, :Hk], dv=self.gv, dgate=self.gg, dbias=self.dbias, dwq=self.dwq, dwk=self.dwk,
                    dtable=self.dtable)


def _reference(st):
    f = to_f64
    q, k, v, g, do = f(st.q), f(st.k), f(st.v), f(st.gate), f(st.dout)
    N, Lq, Lk, H, Hk, d = st.shape
    pq, pk = (np.broadcast_to(p.cpu().numpy(), (N, p.numel())) for p in (st.pos_q, st.pos_k))
    wq, wk = f(st.wq), f(st.wk)
    r = {}
    r["rq"], r["rk"] = (ro.forward(x, p, st.freq, norm=True, w=w) for x, p, w in ((q, pq, wq), (k, pk, wk)))
    e = st.edges.cpu().numpy()
    r["bias"] = rl.forward(pq[:1], pk[:1], e, f(st.table))
    rq, rk, b, m = _bf(r["rq"]), _bf(r["rk"]), _bf(r["bias"]), st.mask.cpu().numpy()
    r["out"], r["lse"], _ = co.forward(rq, rk, v, g, b, m)
    gq, gk, r["dv"], r["dgate"], r["dbias"] = co.backward(rq, rk, v, g, b, m, do)
    r["dq"], r["dwq"] = ro.backward(gq, q, pq, st.freq, norm=True, w=wq)
    r["dk"], r["dwk"] = ro.backward(gk, k, pk, st.freq, norm=True, w=wk)
    r["dtable"] = rl.backward(pq[:1], pk[:1], e, r["dbias"])
    count = rl.backward(pq[:1], pk[:1], e, np.ones_like(r["dbias"]))
    slack = {"dtable": 2e-2 * np.sqrt(count) * np.sqrt(np.sum(r["dbias"] ** 2, (0, 2, 3)))[:, None]}
    for n, gr_, x, p in (("dwq", gq, q, pq), ("dwk", gk, k, pk)):
        t = ro.rotate(gr_, p, st.freq, False, 1.0, True) * x * ro.rstd(x, 1e-6)
        slack[n] = 2e-2 * np.sqrt(t.shape[0] * t.shape[1] * t.shape[2]) * np.sqrt(np.sum(t * t, (0, 1, 2)))
    return r, slack


def test_training_step_eager_and_captured():
    st = _Step()
    s, cache = torch.cuda.Stream(), gr.GraphCache(capacity=2)
    for replay in range(3):
        for t in (st.qg, st.kv, st.dout):
            t.normal_()
        st.table.normal_(0, 0.3)
        st.mask.random_(0, 2)
        st.mask[:, 3] = 1
        torch.cuda.synchronize()
        cache.run(1, st.first, s)
        s.synchronize()
        st.dbias32.copy_(st.dbias)                                     # relpos_bias_bwd sums fp32
        torch.cuda.synchronize()
        cache.run(2, st.second, s)
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in st.outputs().items()}
        with torch.cuda.stream(s):
            st.first(None)
            st.dbias32.copy_(st.dbias)
            st.second(None)
        torch.cuda.synchronize()
        for name, t in st.outputs().items():
            assert torch.equal(t, got[name]), name                     # a replay gives the eager call's bits
        ref, slack = _reference(st)
        for name, want in ref.items():
            have = to_f64(got[name])
            if name in slack:
                assert (np.abs(have - want) <= slack[name]).all(), name
            else:
                off = np.linalg.norm(have - want) / np.linalg.norm(want)
                assert off <= 2e-2, (name, off)


def test_single_tokens_follow_the_whole():
    """One token at a time, at its own position, gives the rows of the whole call."""
    N, L, Lk, H, Hk, d = 2, 9, 300, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    q, k, v = r(N, L, H, d), r(N, Lk, Hk, d), r(N, Lk, Hk, d)
    w, steps = torch.rand(d, generator=g, device="cuda") + 0.5, rope.rope_steps(rope.rope_frequencies(d))
    pos = torch.arange(100, 100 + L, dtype=torch.int32, device="cuda")
    pk = torch.arange(Lk, dtype=torch.int32, device="cuda")
    edges = rp.relpos_edges_log(16, 128)
    table = torch.randn(H, edges.numel() + 1, generator=g, device="cuda")
    whole_q, rk = rope.rope_fwd(q, pos, steps, k=k, pos_k=pk, norm=True, weight_q=w, weight_k=w)
    bias = rp.relpos_bias_fwd(pos.view(1, -1), pk.view(1, -1), edges, table)
    whole, lse = cross.cross_attn_fwd(whole_q, rk, v, None, bias)
    for t in range(L):
        qt, _ = rope.rope_fwd(q[:, t:t + 1], pos[t:t + 1], steps, norm=True, weight_q=w)
        bt = rp.relpos_bias_fwd(pos[t:t + 1].view(1, 1), pk.view(1, -1), edges, table)
        ot, lt = cross.cross_attn_fwd(qt, rk, v, None, bt)
        assert torch.equal(qt, whole_q[:, t:t + 1]) and torch.equal(bt, bias[:, :, t:t + 1])
        # another order of the sums over the keys: the probabilities' rounding (2^-8 of sum p |v|, |v| < 6) and the result's
        assert float((ot.float() - whole[:, t:t + 1].float()).abs().max()) <= 2 * 2.0 ** -8 * 6
        assert float((lt - lse[:, :, t:t + 1]).abs().max()) <= 1e-4
