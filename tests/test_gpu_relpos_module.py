"""The relative position bias where it is used: the attention module step with
it, its gradient out of the attention's backward, and a training step whose
matrices go through the Muon step and whose vectors and bias table go through
Adam, eager and captured.

Tolerances.  Module chain: 2e-2 normwise per tensor, as in the module test
without the bias (bf16 hand-offs; one more rounding of the bias, 2^-8 of it).
The table's gradient sums the attention's dbias over n entries, so an error of
norm e in it moves an entry by at most sqrt(n) e (Cauchy-Schwarz): 2e-2 sqrt(n)
|dbias of the head|.  Against the sums of the GPU's own dbias it is the fp32
sums' n 2^-24 of the magnitudes.  Muon: 24000 (2^-21 + sqrt(K) 2^-24) of the
update for any spectrum (see test_gpu_muon), times lr and the update's scale.
"""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import muon_oracle as mo
from oracle import relpos_oracle as ro
from paper_2404_11068_amd import graph as gr
from paper_2404_11068_amd import optim as op
from paper_2404_11068_amd import relpos as rp
from paper_2404_11068_amd import workloads as W
from tests.parity_util import to_f64

pytestmark = pytest.mark.gpu


def _bf(x):
    return W.as_float64(W._store(np.asarray(x, dtype=np.float64), "bf16"), "bf16")


def _rel(got, ref):
    return float(np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-30))


def test_a_table_of_zeros_changes_nothing():
    edges = rp.relpos_edges_clip(8)
    a, b = gr.MSARowAttentionStep(N=3, L=64, seed=5), gr.MSARowAttentionStep(N=3, L=64, seed=5, relpos_edges=edges)
    b.relpos_table.zero_()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for step in (a, b):
        step.record(s)
    torch.cuda.synchronize()
    assert a.key() != b.key() and "d_relpos" not in a.outputs()
    for name, t in a.outputs().items():
        assert torch.equal(t, b.outputs()[name]), name


def test_refuses_wrong_edges():
    for edges in (torch.zeros(3, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda"),
                  torch.zeros(8, dtype=torch.int32, device="cuda")[::2]):
        with pytest.raises(ValueError):
            gr.MSARowAttentionStep(N=1, L=32, relpos_edges=edges)


@pytest.mark.parametrize("N,L,kind", [(4, 64, "clip"), (2, 96, "log")])
def test_module_step_with_relpos_matches_oracle_chain(N, L, kind):
    print("\n[case] module with relpos N=%d L=%d %s" % (N, L, kind), flush=True)
    edges = rp.relpos_edges_clip(32) if kind == "clip" else rp.relpos_edges_log(16, 128)
    step = gr.MSARowAttentionStep(N=N, L=L, seed=22, relpos_edges=edges)
    s, cache = torch.cuda.Stream(), gr.GraphCache(capacity=2)
    rng = np.random.default_rng(3)
    H, HD = step.H, step.H * step.d
    for replay in range(3):  # other residue numbers and tables in the same graph
        pos = np.cumsum(1 + (rng.random((1, L)) < 0.1) * rng.integers(0, 40, (1, L)), 1).astype(np.int32)
        step.relpos_pos.copy_(torch.from_numpy(pos))
        step.relpos_table.normal_()
        torch.cuda.synchronize()
        cache.run(step.key(), step.record, s)
        torch.cuda.synchronize()
        got = {k: to_f64(v) for k, v in step.outputs().items()}

        f, e = to_f64, edges.cpu().numpy()
        pair = _bf(oracle.pair_bias_forward(f(step.z), f(step.ln_z_w), f(step.ln_z_b), f(step.w_bias)))
        bias = _bf(ro.forward(pos, pos, e, f(step.relpos_table), base=pair))
        q, k, v, g = (_bf(o).reshape(N, L, H, step.d) for o in oracle.ln_proj_forward(
            f(step.m), f(step.ln_m_w), f(step.ln_m_b), f(step.w_qkvg), f(step.b_qkvg), n_proj=4))
        mask = np.ones((N, L), np.uint8)
        o, _ = oracle.forward(q, k, v, g, bias, mask, rows_per_bias=N)
        d_o, _, _ = oracle.linear_backward(_bf(o).reshape(N, L, HD), f(step.w_out), [f(step.d_m_out)])
        dq, dk, dv, dg, dbias = oracle.backward(q, k, v, _bf(d_o).reshape(N, L, H, step.d), g, bias, mask,
                                                rows_per_bias=N)
        for name, r in (("bias", bias), ("out", o), ("dq", dq), ("dk", dk), ("dv", dv), ("dg", dg), ("dbias", dbias)):
            assert _rel(got[name].reshape(r.shape), r) <= 2e-2, (name, replay)
        n = np.bincount(ro.buckets(pos, pos, e).reshape(-1), minlength=len(e) + 1)
        size = np.linalg.norm(dbias[0].reshape(H, -1), axis=1)
        assert (np.abs(got["d_relpos"] - ro.backward(pos, pos, e, dbias)) <= 2e-2 * size[:, None] * np.sqrt(n)).all()
        own, mag = ro.backward(pos, pos, e, got["dbias"]), ro.backward(pos, pos, e, np.abs(got["dbias"]))
        assert (np.abs(got["d_relpos"] - own) <= (n + 1) * 2.0 ** -24 * mag).all()


def _training(step):
    """fp32 parameters and gradients of the step: (Muon's matrices, Adam's vectors and table)."""
    mats = {n: getattr(step, n).float() for n in ("w_qkvg", "w_bias", "w_out")}
    vecs = {n: getattr(step, n).clone() for n in ("ln_m_w", "ln_m_b", "ln_z_w", "ln_z_b", "b_qkvg", "b_out",
                                                  "relpos_table")}
    grads = {"relpos_table": step.d_relpos, "b_qkvg": step.db_qkvg, "b_out": step.db_out}
    grad = lambda n: grads.get(n, getattr(step, "d" + n, None))
    adam = op.FusedAdamSWA(list(vecs.values()), [grad(n) for n in vecs], lr=1e-2)
    muon = op.FusedMuonSWA(list(mats.values()), [grad(n) for n in mats], lr=2e-2, weight_decay=0.01)
    return adam, muon


def test_training_steps_eager_and_captured():
    print("\n[case] module, relpos, adam and muon", flush=True)
    edges = rp.relpos_edges_log(16, 64)
    A, B = (gr.MSARowAttentionStep(N=4, L=64, seed=31, relpos_edges=edges) for _ in range(2))
    (adam_a, muon_a), (adam_b, muon_b) = _training(A), _training(B)
    s, cache = torch.cuda.Stream(), gr.GraphCache(capacity=1)

    def run(step, adam, muon, stream):
        step.record(stream)
        adam.step(max_norm=0.5, stream=stream, step=7)
        muon.step(grad_scale=adam.scale, stream=stream)

    for it in range(4):
        for t in (A, B):
            t.m.copy_(torch.randn(t.m.shape, generator=torch.Generator().manual_seed(it)).to(t.m.dtype))
        before = [(p.clone(), m.clone(), w.clone()) for p, m, w in zip(muon_a.params, muon_a.momentum, muon_a.swa)]
        torch.cuda.synchronize()
        run(A, adam_a, muon_a, torch.cuda.current_stream())
        torch.cuda.synchronize()
        cache.run(B.key(), lambda st: run(B, adam_b, muon_b, st), s)
        torch.cuda.synchronize()
        for name, t in A.outputs().items():
            assert torch.equal(t, B.outputs()[name]), (it, name)
        for x, y in zip(adam_a.params + muon_a.params + muon_a.momentum + muon_a.swa,
                        adam_b.params + muon_b.params + muon_b.momentum + muon_b.swa):
            assert torch.equal(x, y) and torch.isfinite(x).all(), it
        scale = float(adam_a.scale)
        for (p, m, w), P, g, M in zip(before, muon_a.params, muon_a.grads, muon_a.momentum):
            up = math.sqrt(max(1.0, p.shape[0] / p.shape[1]))
            rp_, rm, _ = mo.muon_step(to_f64(p), to_f64(g), to_f64(m), to_f64(w), lr=2e-2, momentum_decay=0.95,
                                      nesterov=True, weight_decay=0.01, swa_decay=0.999, update_scale=up, grad_scale=scale)
            assert np.linalg.norm(to_f64(M) - rm) <= 2.0 ** -21 * (np.linalg.norm(to_f64(m)) + scale * np.linalg.norm(to_f64(g))), it
            e = 2.0 ** -21 + math.sqrt(max(p.shape)) * 2.0 ** -24
            assert np.linalg.norm(to_f64(P) - rp_) <= 2e-2 * up * 24000 * e + 2.0 ** -22 * np.linalg.norm(rp_), it
        for t, (adam, muon) in ((A, (adam_a, muon_a)), (B, (adam_b, muon_b))):  # the next step's weights
            for n, p in zip(("w_qkvg", "w_bias", "w_out"), muon.params):
                getattr(t, n).copy_(p)
            for n, p in zip(("ln_m_w", "ln_m_b", "ln_z_w", "ln_z_b", "b_qkvg", "b_out", "relpos_table"), adam.params):
                getattr(t, n).copy_(p)
