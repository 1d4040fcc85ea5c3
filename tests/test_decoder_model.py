"""Rotary positions and causal attention as model operators: the oracle against torch, the library's profile, plan
and checks against the oracle's, and sliced forwards on the GPU."""
import numpy as np
import pytest
import torch

import oracle
import oracle.plan as op_
import synth
from tests.serving_ref import rotate
from tests.helpers import TOL, boundary_codecs, rel_err

import paper_2404_02445_amd as P
from paper_2404_02445_amd import _lib as L

SMALL = dict(batch=2, seq=70, layers=2, hidden=96, heads=4, kv_heads=2, head_dim=32, ffn=128, vocab=101)
VARIANTS = {
    "plain": {},
    "half_part_linear": dict(rotary=dict(rot_dim=16, scaling="linear", factor=4.0)),
    "pairs_yarn": dict(rotary=dict(layout="interleaved", scaling="yarn", factor=8.0, context=64.0), heads=6, kv_heads=1),
    "f32_ntk": dict(dtype="f32", rotary=dict(scaling="ntk", factor=2.0), heads=3, kv_heads=3),
}


def model(**kw):
    return synth.build(8, **{**SMALL, **kw})


@pytest.mark.parametrize("kw,m", [(dict(), 1.0), (dict(rot_dim=20), 1.0), (dict(layout="interleaved", scaling="linear", factor=3.0), 1.0),
                                  (dict(scaling="ntk", factor=4.0, base=5000.0), 1.0),
                                  (dict(scaling="yarn", factor=4.0, context=512.0), 0.1 * np.log(4.0) + 1), (dict(mscale=0.5), 0.5)])
def test_oracle_rotary(kw, m):
    x = np.random.default_rng(1).standard_normal((2, 9, 5 * 32))
    got = oracle.rotary(x, 3, 32, **kw).reshape(2, 9, 5, 32)
    a = {k: v for k, v in kw.items() if k not in ("rot_dim", "layout", "mscale")}
    for b in range(2):
        ref, _ = rotate(torch.from_numpy(x[b].reshape(9, 5, 32)), torch.arange(9), kw.get("rot_dim", 32), kw.get("layout", "half"), m, **a)
        assert np.abs(got[b, :, :3] - ref[:, :3].numpy()).max() < 1e-12
        assert np.array_equal(got[b, :, 3:], x[b].reshape(9, 5, 32)[:, 3:])


def test_oracle_rotary_depends_on_the_difference_of_positions():
    q, k = np.random.default_rng(2).standard_normal((2, 1, 1, 64))
    dots = []
    for at in (0, 7, 30):
        rows = np.zeros((1, at + 4, 64))
        rows[0, at], rows[0, at + 3] = q, k
        t = oracle.rotary(rows, 1, 64)
        dots.append(t[0, at] @ t[0, at + 3])
    assert np.allclose(dots, dots[0], atol=1e-12)


def test_oracle_causal_attention_against_torch():
    x = torch.from_numpy(np.random.default_rng(3).standard_normal((2, 33, 8 * 16)))
    t = x.view(2, 33, 8, 16).transpose(1, 2)
    ref = torch.nn.functional.scaled_dot_product_attention(t[:, :4], t[:, 4:6].repeat_interleave(2, 1), t[:, 6:].repeat_interleave(2, 1),
                                                           is_causal=True, scale=0.3)
    got = oracle.causal_attention(x.numpy(), 4, 2, 16, 0.3)
    assert np.abs(got - ref.transpose(1, 2).reshape(2, 33, 64).numpy()).max() < 1e-12


@pytest.mark.parametrize("name", VARIANTS)
def test_profile_and_plan_equal_the_oracles(name):
    m = model(**VARIANTS[name])
    sm = P.SlicedModel(m, device="cpu")
    ref = op_.layer_profiles(m)
    assert [tuple(g) for g in sm.profile()] == [(r.mem_bytes, r.time_s, r.out_bytes, r.rd_width) for r in ref]
    sl, pl = m.slicing, sm.plan()
    po = op_.plan_slices(ref, op_.PlanOpts(n_slices=sl["n_slices"], allowed_cut=sl["allowed_cut"], elim_tau=sl["elim_tau"],
                                           k_override=sl["k_override"]))
    assert (pl.slice_end, pl.k, pl.cost, pl.t_tau) == (po.slice_end, po.k, po.cost, po.t_tau)
    flop = [op_.op_profile(m, o)[2] for o in m.ops if o["kind"] == "causal_attention"]
    s, h, d = 70, VARIANTS[name].get("heads", 4), 32
    assert flop == [4 * 2 * h * d * (s * (s + 1) // 2)] * 2


def create_error(change, **kw):
    m = model(**kw)
    change(m)
    with pytest.raises(P.MoparError) as e:
        P.SlicedModel(m, device="cpu")
    return e.value.status


def test_create_refuses():
    rot, att = (lambda m, k=kind: next(o for o in m.ops if o["kind"] == k) for kind in ("rotary", "causal_attention"))
    for change, want in [(lambda m: rot(m).update(heads=0), L.MOPAR_E_SHAPE), (lambda m: rot(m).update(heads=9), L.MOPAR_E_SHAPE),
                         (lambda m: rot(m).update(head_dim=40), L.MOPAR_E_SHAPE), (lambda m: rot(m).update(rotary=dict(rot_dim=3)), L.MOPAR_E_ARG),
                         (lambda m: rot(m).update(rotary=dict(base=0.1)), L.MOPAR_E_ARG), (lambda m: rot(m).update(head_dim=4, heads=2), L.MOPAR_E_UNSUPPORTED),
                         (lambda m: att(m).update(heads=5), L.MOPAR_E_SHAPE), (lambda m: att(m).update(kv_heads=0), L.MOPAR_E_SHAPE),
                         (lambda m: att(m).update(kv_heads=3, heads=2), L.MOPAR_E_SHAPE), (lambda m: att(m).update(head_dim=64), L.MOPAR_E_SHAPE),
                         (lambda m: att(m).update(scale=0.0), L.MOPAR_E_ARG), (lambda m: att(m).update(scale=float("nan")), L.MOPAR_E_ARG)]:
        assert create_error(change) == want
    assert create_error(lambda m: None, head_dim=48, hidden=96) == L.MOPAR_E_UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("name", VARIANTS)
def test_sliced_forward(name):
    m = model(**VARIANTS[name])
    x = synth.make_input(m)
    xd = torch.from_numpy(x).cuda()
    sm = P.SlicedModel(m)
    plan = sm.plan()
    cuts = plan.slice_end[:-1]
    assert len(cuts) == 2
    _, cw = boundary_codecs(m, cuts)
    codecs, keep = sm.codecs(plan, "ae", cw)
    ws = sm.alloc_workspace(plan)
    ws.fill_(0xFF)
    out = sm.forward(plan, xd, sm.alloc_output(), codecs, sm.alloc_codes(plan, codecs), ws)
    ref = oracle.forward(m, x, k=plan.k, cuts=cuts, codecs=cw)
    assert rel_err(out.float().cpu().numpy(), ref) <= TOL[m.dtype]
    # raw hand-off, no cuts, the static workspace and the pipeline: the same bits
    raw, keep = sm.codecs(plan, "raw")
    a = sm.forward(plan, xd, sm.alloc_output(), raw, sm.alloc_codes(plan, raw), ws)
    n = len(m.layers)
    whole = P.make_plan(n, [n - 1], [1] * n)
    b = sm.forward(whole, xd, sm.alloc_output(), None, None, sm.alloc_workspace(whole))
    c = sm.forward_static(whole, xd, sm.alloc_output())
    pipe = sm.pipeline(plan, "raw", None, depth=2, replicas=1, stream_per_slice=False)
    pipe.use_graphs(True)
    o = sm.alloc_output()
    torch.cuda.synchronize()
    for _ in range(3):
        o.zero_()
        torch.cuda.synchronize()
        pipe.submit(xd, o)
        pipe.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(a, o)


@pytest.mark.gpu
def test_longer_than_the_bidirectional_attention_and_timed():
    m = model(batch=1, seq=300, head_dim=128, heads=2, kv_heads=1, layers=1)
    x = synth.make_input(m)
    sm = P.SlicedModel(m)
    n = len(m.layers)
    plan = P.make_plan(n, [n - 1], [1] * n)
    sm.set_timing(True)
    out = sm.forward(plan, torch.from_numpy(x).cuda(), sm.alloc_output(), None, None, sm.alloc_workspace(plan))
    ops, _ = sm.op_times()
    assert all(t > 0 for t in ops)
    assert rel_err(out.float().cpu().numpy(), oracle.forward(m, x)) <= TOL["bf16"]


@pytest.mark.gpu
def test_a_model_s_prompt_equals_the_serving_calls():
    """The two operators in a model give what mopar_rotary_apply and mopar_attention_prompt give on the same rows."""
    b = synth._Builder("attn", "bf16", 3, 5)
    ids = b.tensor((3, 90), "i32")
    b.new_layer("embed")
    x = b.embed(ids, 270, 8 * 64, "src", -1.0, 1.0)
    b.new_layer("attn")
    y = b.rotary(x, 6, 64, "rot", dict(layout="interleaved"))
    m = b.finish(b.causal_attention(y, 4, 2, 64, "att"), 1)
    xi = torch.arange(270, dtype=torch.int32, device="cuda").reshape(3, 90)
    sm = P.SlicedModel(m)
    plan = P.make_plan(2, [1], [1, 1])
    out = sm.forward(plan, xi, sm.alloc_output(), None, None, sm.alloc_workspace(plan))
    rows = torch.from_numpy(m.weights["src.table"]).to(torch.bfloat16).cuda().view(270, 8, 64)
    pos = torch.arange(90, dtype=torch.int32, device="cuda").repeat(3)
    qk = torch.empty(270, 6, 64, device="cuda", dtype=torch.bfloat16)
    P.mopar_rotary_apply(P.Rotary(64, layout="interleaved"), rows[:, :6], qk, pos)
    got = torch.empty(270, 4, 64, device="cuda", dtype=torch.bfloat16)
    off = torch.tensor([0, 90, 180, 270], dtype=torch.int32, device="cuda")
    P.mopar_attention_prompt(qk[:, :4], qk[:, 4:], rows[:, 6:], got, off, 90)
    assert torch.equal(out.view(270, 4, 64), got)
