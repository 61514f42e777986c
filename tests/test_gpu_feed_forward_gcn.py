"""The training step with gated feed-forward blocks on the sampled layers and AdamW: gradients against 64-bit automatic differentiation, and the step's arithmetic against 64
bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import plain_training as plain
from paper_2101_07706_amd import synth

RTOL, ATOL = 1e-4, 1e-5      # of an entry, and of the largest one


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2101_07706_amd import csgs, pipeline, residual_gcn
    csgs.lib()
    return csgs, pipeline, residual_gcn


def close(got, want, what):
    got, want = got.double().cpu(), want.detach()
    tol = RTOL * want.abs() + ATOL * want.abs().max() + 1e-30
    worst = ((got - want).abs() / tol).max().item()
    assert worst <= 1.0, f"{what}: error {worst:.2f} times its tolerance"


def reference(net, G):
    """Gradients in float64 of sum(G . logits), and the logits, through the adjacency the step sampled."""
    c = lambda t: t.detach().double().cpu()
    p = {k: c(v).requires_grad_(True) for k, v in net.params.items()}
    counts = [net.batch] + [int(lb.n_next) for lb in net.lbs]
    ids = [net.ids[net.at[l]:net.at[l] + counts[l]].long().cpu() for l in range(net.L + 1)]
    table = c(net.table).requires_grad_(True)
    x = [net.scale * table[i] for i in ids]

    def layer_norm(v, w, b):
        m = v.mean(1, keepdim=True)
        return (v - m) / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + 1e-5) * w + b

    u = layer_norm(x[-1], p["bottom.pre_w"], p["bottom.pre_b"])
    for l in range(net.L - 1, -1, -1):
        lb = net.lbs[l]
        ptr, col, val = lb.adj_rowptr.cpu().long(), lb.adj_col.cpu().long(), c(lb.adj_val)
        P = torch.zeros(counts[l], counts[l + 1], dtype=torch.float64)
        for r in range(counts[l]):
            P[r, col[ptr[r]:ptr[r + 1]]] = val[ptr[r]:ptr[r + 1]]
        z = P @ torch.relu(u)
        g = z @ p[f"{l}.wg"]
        h = (g * torch.sigmoid(g) * (z @ p[f"{l}.wu"])) @ p[f"{l}.wd"] + p[f"{l}.bd"]
        n = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5) * p[f"{l}.post_w"] + p[f"{l}.post_b"]
        u = layer_norm(net.beta * x[l] + torch.sigmoid(p[f"{l}.gate"]) * n, p[f"{l}.pre_w"], p[f"{l}.pre_b"])
    logits = u @ p["w_out"]
    (logits * c(G)).sum().backward()
    return logits, {k: v.grad for k, v in p.items()}, table.grad


def make(residual_gcn, pipeline, width, L=2, seed=3, **kw):
    g = synth.make_sbm(1500, 4, 0.02, 0.002, 5)
    dg = pipeline.DeviceGraph(g)
    net = residual_gcn.ResidualGCN(dg, width, 5, L, 100, 128, 4.0, g.nnz, seed=seed, **kw)
    for k, v in net.params.items():       # nothing at its neutral value
        v.add_(torch.randn(v.shape, generator=torch.Generator().manual_seed(len(k))).to(v.device), alpha=0.1)
    S0 = torch.from_numpy(synth.make_batch(g, 100, 1)).to(dg.device)
    return g, net, S0


@pytest.mark.parametrize("width,ffn,L", [(64, 256, 2), (30, 77, 1), (100, 130, 3)])
def test_gradients(env, width, ffn, L):
    csgs, pipeline, residual_gcn = env
    g, net, S0 = make(residual_gcn, pipeline, width, L, ffn=ffn)
    for it in range(2):                   # the second step finds the first one's leftovers in every buffer
        logits = net.forward(S0, it).clone()
        G = torch.randn(logits.shape, generator=torch.Generator().manual_seed(it)).to(logits.device) / 100
        net.backward(G)
        torch.cuda.synchronize()
        assert all(int(lb.status) == 0 for lb in net.lbs)
        want, grads, table = reference(net, G)
        close(logits, want, "logits")
        for k, v in net.grads.items():
            close(v, grads[k], k)
        n = int(net.table_count)
        close(net.table_rows[:n], table[net.table_ids[:n].long().cpu()], "table")


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ffn", [0, 96])
def test_adamw_steps(env, bits, ffn):
    """What a step does to weights and states follows from its own gradients."""
    csgs, pipeline, residual_gcn = env
    g, net, S0 = make(residual_gcn, pipeline, 48, ffn=ffn, optimizer="adamw", state_bits=bits, lr=0.01, max_norm=0.05)
    lr, wd = float(np.float32(0.01)), float(np.float32(0.01))
    max_norm = float(np.float32(0.05))
    G = torch.randn(100, 5, generator=torch.Generator().manual_seed(0)).to(S0.device) / 100
    for t in range(1, 4):
        net.forward(S0, t)
        net.backward(G)
        old = {k: v.cpu() for k, v in net.params.items()}
        states = {k: {n: x.cpu() for n, x in s.items()} for k, s in net.states.items()}
        table = net.table.cpu()
        net.clip()
        net.descend()
        n = int(net.table_count)
        total = math.sqrt(math.fsum([float((v.double() ** 2).sum()) for v in net.grads.values()] + [float((net.table_rows[:n].double() ** 2).sum())]))
        assert int(net.steps_taken) == t and int(net.status) == 0 and abs(float(net.norm) - total) <= 2.0 ** -23 * total
        c = min(1.0, max_norm / (total + 1e-6))
        ids = net.table_ids[:n].long().cpu()
        for k in list(net.params) + ["table"]:
            s = states[k]
            rows = ids if k == "table" else slice(None)
            small = "m_exp" in s
            assert small == (bits == 8 and (k == "table" or net.params[k].dim() == 2))
            shape = s["m"].shape
            m = plain.decode(s["m"], s["m_exp"], False) if small else s["m"].double()
            v = plain.decode(s["v"], s["v_exp"], True) if small else s["v"].double()
            p = (table if k == "table" else old[k]).reshape(shape)
            grad = (net.table_rows[:n] if k == "table" else net.grads[k]).cpu().reshape(-1, shape[1])
            decay = wd if k != "table" and net.params[k].dim() == 2 else 0.0
            wp, wm, wv, change = plain.adamw(p[rows], grad, m[rows], v[rows], t, lr, 0.9, 0.999, float(np.float32(1e-8)), decay, c)
            got = (net.table if k == "table" else net.params[k]).cpu().reshape(shape)
            assert bool(((got[rows].double() - wp).abs() <= 2.0 ** -24 * (2 * wp.abs() + 14 * change) + 1e-38).all()), k
            new = {q: x.cpu() for q, x in net.states[k].items()}
            if small:
                for q, x, second in (("m", wm, False), ("v", wv, True)):
                    code, exps = plain.encode(x.float(), second)
                    assert torch.equal(new[q][rows], code) and torch.equal(new[q + "_exp"][rows], exps), (k, q)
            else:
                assert bool(((new["m"][rows].double() - wm).abs() <= (2.0 ** -24 + 2.0 ** -45) * wm.abs() + 2.0 ** -149).all()), k
            if k == "table":
                rest = torch.ones(shape[0], dtype=torch.bool)
                rest[ids] = False
                assert torch.equal(got[rest], p[rest]) and all(torch.equal(new[q][rest], s[q][rest]) for q in s)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_an_adamw_step_without_finite_gradients_changes_nothing(env, bad):
    csgs, pipeline, residual_gcn = env
    g, net, S0 = make(residual_gcn, pipeline, 48, ffn=64, optimizer="adamw", state_bits=8, lr=0.01)
    G = torch.randn(100, 5, device=S0.device) / 100

    def step(G, it):
        net.forward(S0, it)
        net.backward(G)
        net.clip()
        net.descend()

    everything = lambda: [net.table.clone()] + [v.clone() for v in net.params.values()] + [x.clone() for s in net.states.values() for x in s.values()]
    step(G, 0)
    before = everything()
    wrong = G.clone()
    wrong[7, 2] = bad
    for it in (1, 2):
        step(wrong, it)
        assert int(net.status) == csgs.ST_NONFINITE_GRAD and int(net.skipped) == it and int(net.steps_taken) == 1
        assert all(torch.equal(a, b) for a, b in zip(before, everything()))
    step(G, 3)
    assert int(net.status) == 0 and int(net.skipped) == 2 and int(net.steps_taken) == 2
    assert all(bool(torch.isfinite(v).all()) for v in net.params.values()) and not torch.equal(before[0], net.table)


def test_steps_repeat_bit_for_bit(env):
    csgs, pipeline, residual_gcn = env
    labels = torch.from_numpy((np.arange(100) % 5).astype(np.int64))
    runs = []
    for _ in range(2):
        g, net, S0 = make(residual_gcn, pipeline, 48, ffn=64, optimizer="adamw", lr=0.01)
        losses = [float(net.step(S0, labels.to(S0.device), it)) for it in range(3)]
        assert all(math.isfinite(x) for x in losses) and int(net.skipped) == 0
        runs.append([net.table] + list(net.params.values()))
    assert all(torch.equal(a, b) for a, b in zip(*runs))
