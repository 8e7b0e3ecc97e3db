"""The orthogonalised update of the library's own model: ppo_gradient, muon_update of the hidden layers' matrices where they lie in the flat vector,
adam_update of everything else, and the shadow that the agents read."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import bf16model as bm  # noqa: E402
from oracle import ppo as oppo  # noqa: E402
from workloads import synthetic as syn  # noqa: E402
from gpu_util import rel_l2  # noqa: E402
from test_gpu_muon import TOL, steps64  # noqa: E402
from test_gpu_parity import _bind_model, _filled_buffer, dev, zeros, g, inst, _keep_device_inputs_alive  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["C2", "C4"])
def test_a_step_of_the_model(g, inst, name):  # noqa: F811
    cfg = syn.get_config(name)
    shape = oppo.ModelShape(cfg.obs_dim, cfg.act_dim, tuple(cfg.hidden))
    theta = syn.make_model_params(cfg.obs_dim, cfg.act_dim, cfg.hidden, 3, policy_head_scale=0.5)
    T, N, rows = 2, 512, 1024
    b, rb, hb = _filled_buffer(g, inst, cfg, T, N, seed=2)
    flat = oppo.flatten_buffer(b)
    pol, _, log_std = oppo.unpack(theta.astype(np.float64), shape)
    z = (flat["act"] - oppo.mlp_forward(flat["obs"].astype(np.float64), pol)[0]) * np.exp(-log_std)
    logp = (-0.5 * z * z - log_std - 0.5 * oppo.LOG_2PI).sum(1)      # of the policy itself: ratios of about 1
    rb.logp.copy_(dev((logp + 0.05 * np.random.default_rng(4).standard_normal(T * N)).astype(np.float32).reshape(T, N)))
    b["adv"], b["ret"] = oppo.gae(b["rew"], b["val"], b["done"], b["last_val"], 0.99, 0.95, True)
    rb.adv.copy_(dev(b["adv"])); rb.ret.copy_(dev(b["ret"]))
    torch.cuda.synchronize()
    hm, (params, shadow, _, _) = _bind_model(g, inst, cfg, theta, rows, "bf16")
    grad, stats = zeros(theta.size), zeros(5)
    matrices, others, at, done = [], [], 0, 0      # (rows, cols, offset); (begin, end) of biases, heads and log_std
    for out_dim in (shape.act_dim, 1):
        dims = shape.layer_dims(out_dim)
        for l, (k, n) in enumerate(dims):
            if l < len(dims) - 1:
                matrices.append((n, k, at))
                if at > done:
                    others.append((done, at))
                done = at + n * k
            at += n * k + n
    others.append((done, theta.size))
    moments, adam_m, adam_v = zeros(theta.size), zeros(theta.size), zeros(theta.size)
    hm_muon = g.gmi_muon_bind(inst, matrices, g.DTYPE_F32)
    idx = dev(np.random.default_rng(3).permutation(T * N)[:rows].astype(np.int32))
    hp = g.ppo_hparams(clip=0.2, c_v=0.5, c_e=0.01, minibatch=rows, lr=1e-3)
    torch.cuda.synchronize()
    g.ppo_gradient(inst, hm, hb, hp, idx, rows, grad, stats)
    g.muon_update(inst, hm_muon, params, moments, grad, g.muon_hparams(lr=0.05))
    for a, e in others:
        g.adam_update(inst, params[a:e], adam_m[a:e], adam_v[a:e], grad[a:e], e - a, hp, 1)
    g.gmi_model_refresh_shadow(inst, hm)
    g.gmi_sync(inst)
    new, gr = params.cpu().double(), grad.cpu().double()
    assert torch.isfinite(new).all()
    for n, k, o in matrices:
        u = gr[o:o + n * k].view(n, k) * (1 + 0.95)      # the first step: m = g, u = g + mu m
        lr = 0.05 * math.sqrt(max(1.0, n / k))
        step = lr * steps64(u, 5)
        old = torch.from_numpy(theta[o:o + n * k]).double().view(n, k)
        got = new[o:o + n * k].view(n, k)
        # the step's own error: each of the five rounds what it starts from to 22 bits, and the directions of small singular values, of which a network's
        # gradient has many, are lengthened by a = 3.4445 in every step that follows; the rounding of the parameters to fp32
        own = TOL["f32"] * float(step.norm()) + lr * 5 * 3.4445 ** 5 * 2.0 ** -22
        assert float((got - (old - step)).norm()) <= own + 2e-7 * float(old.norm()), (n, k)
    for a, e in others:      # the first step of Adam: lr g / (|g| + eps), what is not 0 moves by about lr
        moved = new[a:e] - torch.from_numpy(theta[a:e]).double()
        assert float(moved.abs().max()) <= 1.001e-3 + 1e-7 and (moved[gr[a:e].abs() > 1e-4] * gr[a:e][gr[a:e].abs() > 1e-4] < 0).all()
    obs = syn.make_initial_state(300, cfg.obs_dim, 5)
    A = cfg.act_dim
    act, logp, val, mu = zeros(300, A), zeros(300), zeros(300), zeros(300, A)
    g.agent_act(inst, hm, dev(obs), 300, 42, 9, 100, act, logp, val, mu)
    g.gmi_sync(inst)
    want_mu, want_val = bm.agent_forward(params.cpu().numpy(), shape, obs)
    assert rel_l2(mu.cpu().numpy(), want_mu) <= 1e-3 and rel_l2(val.cpu().numpy(), want_val) <= 1e-3
    g.gmi_muon_destroy(hm_muon)
    g.gmi_model_destroy(hm)
    g.gmi_buffer_destroy(hb)
