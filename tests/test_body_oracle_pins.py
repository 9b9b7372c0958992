"""Pins for the student-body oracle: closed forms, torch's own types and float64 autograd, central differences."""
import numpy as np
import pytest
import torch

from oracle import body_oracle as O


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_record_error_bound_idempotence_and_smallest_exponent(fmt):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 70)) * 10.0 ** rng.integers(-30, 30, (40, 1))
    x[3] = 0.0
    v = O.record_values(x, fmt)
    e, _ = O.record_exponents(x, fmt)
    assert np.array_equal(O.record_values(v, fmt), v)                      # values of a record are kept as they are
    for g in range(3):
        part, kept = x[:, 32 * g:32 * g + 32], v[:, 32 * g:32 * g + 32]
        top = np.abs(part).max(axis=1)
        bound = top[:, None] / 127 if fmt == "int8" else np.abs(part) / 16 + top[:, None] * 2.0 ** -17
        assert (np.abs(part - kept) <= bound).all()
        assert (top <= O.Q[fmt] * 2.0 ** e[:, g]).all()
        assert ((top > O.Q[fmt] * 2.0 ** (e[:, g] - 1)) | (e[:, g] == -126)).all()
    assert not v[3].any() and (e[3] == -126).all()


def test_record_by_hand():
    x = np.zeros((2, 32))
    x[0, :4] = [127.0, 0.5, 1.5, -2.5]                                     # step 1: ties go to even
    x[1, :3] = [128.0, 1.0, 3.0]                                           # step 2
    v = O.record_values(x, "int8")
    assert v[0, :4].tolist() == [127.0, 0.0, 2.0, -2.0] and v[1, :3].tolist() == [128.0, 0.0, 4.0]
    x[0, 1] = np.inf
    assert np.isnan(O.record_values(x, "int8")[0]).all() and np.isfinite(O.record_values(x, "int8")[1]).all()


def test_e4m3_rounding_is_torchs():
    q = np.concatenate([np.linspace(-448, 448, 20001), 2.0 ** np.linspace(-12, 8.8, 5000)])
    want = torch.tensor(q, dtype=torch.float32).to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(O.round_e4m3(q.astype(np.float32).astype(np.float64)), want)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_is_torchs_and_its_gradient(act):
    g0, u0, dh = (torch.randn(9, 13, dtype=torch.float64, generator=torch.Generator().manual_seed(s)) * 3 for s in (1, 2, 3))
    g, u = g0.clone().requires_grad_(True), u0.clone().requires_grad_(True)
    a = torch.nn.functional.silu(g) if act == "silu" else torch.nn.functional.gelu(g, approximate="tanh")
    h = a * u
    h.backward(dh)
    np.testing.assert_allclose(O.gated_forward(g0.numpy(), u0.numpy(), act), h.detach().numpy(), rtol=1e-12, atol=1e-14)
    dg, du = O.gated_backward(g0.numpy(), u0.numpy(), dh.numpy(), act)
    np.testing.assert_allclose(dg, g.grad.numpy(), rtol=1e-10, atol=1e-13)
    np.testing.assert_allclose(du, u.grad.numpy(), rtol=1e-10, atol=1e-13)


@pytest.mark.parametrize("kind", ["none", "channel", "token"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
def test_norm_gradient_is_autograds_and_differences(kind, post, pre):
    T, H, eps, offset, alpha, beta = 5, 7, 1e-3, 1.0, 0.7, 1.3
    rng = np.random.default_rng(4)
    v = {n: rng.standard_normal(s) for n, s in dict(r=(T, H), b=(T, H), w1=(H,), w2=(H,), dy=(T, H), dx=(T, H)).items()}
    v["gate"] = rng.standard_normal(H if kind == "channel" else T)
    w1, w2 = (v["w1"] if post else None), (v["w2"] if pre else None)
    args = dict(w1=w1, w2=w2, gate=v["gate"], kind=kind, offset=offset, alpha=alpha, beta=beta)
    f = O.norm_forward(v["r"], v["b"], eps=eps, **args)
    o = O.norm_backward(v["dy"] if pre else None, v["dx"], v["b"], f["x"], f["rho1"], f["rho2"], **args)

    t = {n: torch.tensor(a, requires_grad=True) for n, a in v.items()}
    rms = lambda z: torch.rsqrt((z * z).mean(1, keepdim=True) + eps)        # noqa: E731
    n = t["b"] * rms(t["b"]) * (t["w1"] + offset) if post else t["b"]
    gate = {"none": 1.0, "channel": t["gate"], "token": t["gate"][:, None]}[kind]
    x = beta * t["r"] + alpha * gate * n
    total = (x * t["dx"].detach()).sum()
    if pre:
        y = x * rms(x) * (t["w2"] + offset)
        np.testing.assert_allclose(f["y"], y.detach().numpy(), rtol=1e-12)
        total = total + (y * t["dy"].detach()).sum()
    total.backward()
    np.testing.assert_allclose(f["x"], x.detach().numpy(), rtol=1e-12)
    for name, grad in (("r", "dr"), ("b", "db"), ("w1", "dw1"), ("w2", "dw2"), ("gate", "dgate")):
        if o[grad] is None:
            assert t[name].grad is None
            continue
        np.testing.assert_allclose(o[grad], t[name].grad.numpy(), rtol=1e-9, atol=1e-12)

    def value(**changed):
        z = dict(v, **changed)
        got = O.norm_forward(z["r"], z["b"], eps=eps, **dict(args, w1=z["w1"] if post else None,
                                                             w2=z["w2"] if pre else None, gate=z["gate"]))
        return (got["x"] * v["dx"]).sum() + ((got["y"] * v["dy"]).sum() if pre else 0.0)
    for name, grad in (("r", "dr"), ("b", "db"), ("w1", "dw1"), ("w2", "dw2"), ("gate", "dgate")):
        if o[grad] is None:
            continue
        at = tuple(rng.integers(0, s) for s in v[name].shape)
        step = np.zeros_like(v[name])
        step[at] = 1e-5
        diff = (value(**{name: v[name] + step}) - value(**{name: v[name] - step})) / 2e-5
        assert abs(diff - o[grad][at]) <= 1e-7 * max(1.0, abs(diff))
