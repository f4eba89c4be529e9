"""GPU tests of the losses' binding: its native wrappers against its general path, what that converts, and what both refuse."""
import math

import pytest
import torch

from paper_2603_16219_amd import losses

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def loaded():
    assert torch.cuda.is_available(), "GPU tests need a device"
    losses.library()
    assert losses._calls is not None


def inputs(B=4, T=6, V=1003, dtype=torch.bfloat16, pad=0):
    g = torch.Generator("cuda").manual_seed(B * V + T + pad)
    x, z = (torch.randn(B, T + pad, V + pad, generator=g, device="cuda").to(dtype)[:, :T, :V] for _ in range(2))
    rows = lambda: torch.randn(B, T, generator=g, device="cuda") - 7
    return dict(x=x, z=z, y=torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32), old=rows(), ref=rows(), adv=rows() + 7,
                mask=torch.rand(B, T, generator=g, device="cuda") < 0.7)


def calls(i, **more):
    """Every call on inputs `i`, as functions without arguments."""
    tau = dict(temperature=0.8)
    stats = losses.token_logprobs(i["x"], i["y"], mask=i["mask"], **tau, want_stats=True)["stats"]
    given = {k: v for k, v in more.items() if k != "grad_logits"}
    return [
        lambda: losses.token_logprobs(i["x"], i["y"], mask=i["mask"], **tau, want_stats=True, **given),
        lambda: {"g": losses.token_logprobs_grad(i["x"], i["y"], stats, i["old"], mask=i["mask"], **tau, grad_scale=2, grad_logits=more.get("grad_logits"))},
        lambda: losses.policy_loss(i["x"], i["y"], i["old"], i["adv"], mask=i["mask"], **tau, reduction="seq_mean", **more),
        lambda: losses.policy_loss(i["x"], i["y"], i["old"], i["adv"][:, 0].contiguous(), mask=i["mask"], ref_logprobs=i["ref"], kl_coef=0.1, **tau, **more),
        lambda: losses.policy_loss(i["x"], i["y"], i["old"], i["adv"], ref_logits=i["z"], kl_coef=1, clip_high=0.3, reduction="sum", grad_scale=0.5, **tau, **more),
        lambda: losses.preference_loss(i["x"], i["y"], mask=i["mask"], ref_logprobs=i["ref"], beta=0.2, label_smoothing=0.1, reduction="sum", **tau, **more),
        lambda: losses.preference_loss(i["x"], i["y"], **more),
    ]


def alike(a, b):
    assert list(a) == list(b)
    for k in a:
        assert (a[k] is None) == (b[k] is None), k
        assert a[k] is None or (a[k].dtype == b[k].dtype and a[k].shape == b[k].shape and torch.equal(a[k], b[k]) and not a[k].requires_grad), k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,T,V,pad", [(4, 6, 1003, 0), (4, 6, 1003, 3), (2, 1, 70001, 0), (2, 1, 999, 1), (4, 60, 4099, 0)])
def test_native_and_general_path_agree(monkeypatch, dtype, B, T, V, pad):
    i = inputs(B, T, V, dtype, pad)
    need = losses.workspace_bytes(losses._make_params(i["x"], i["y"], 1.0))
    for more in ({}, {"workspace": torch.empty(need, dtype=torch.uint8, device="cuda")}, {"grad_logits": torch.empty(B, T + 2, V + 1, dtype=dtype, device="cuda")[:, 1:-1, :V]}):
        if pad and "grad_logits" in more:
            i["x"].requires_grad_()
        for call in calls(i, **more):
            taken = []
            with monkeypatch.context() as m:
                m.setattr(losses, "_native", lambda *a, f=losses._native: taken.append(f(*a)) or taken[-1])
                native = call()
            assert taken[-1] is not None
            native = {k: None if v is None else v.clone() for k, v in native.items()}
            with monkeypatch.context() as m:
                m.setattr(losses, "_calls", None)
                alike(native, call())


def test_what_is_given_for_outputs_comes_back():
    i = inputs()
    for call in calls(i, grad_logits=i["x"])[1:]:
        i["x"].copy_(i["z"])
        out = call()
        assert out.get("grad_logits", out.get("g")) is i["x"]


def test_what_has_to_be_converted():
    i = inputs()
    want = [c() for c in calls(i)]
    j = dict(i)
    j.update(y=i["y"].long(), old=i["old"].double(), ref=i["ref"].double(), adv=i["adv"].double(), mask=i["mask"].T.contiguous().T)
    for a, b in zip(want, [c() for c in calls(j)]):
        alike(a, b)
    j.update(y=i["y"].cpu(), old=i["old"].cpu(), ref=i["ref"].cpu(), adv=i["adv"].T.contiguous().T, mask=i["mask"].byte() * 7)
    for a, b in zip(want, [c() for c in calls(j)]):
        alike(a, b)
    y = i["y"].long()
    y[0, 0] += 2**32  # not the valid id that its lower half is
    assert losses.token_logprobs(i["x"], y)["logprobs"].isnan().sum() == 1


def test_a_reference_whose_strides_differ_where_they_mean_nothing():
    i = inputs(B=3, T=1, V=515)
    want = losses.policy_loss(i["x"], i["y"], i["old"], i["adv"], ref_logits=i["z"], kl_coef=0.1)
    z = torch.as_strided(torch.empty(3 * 515, dtype=i["z"].dtype, device="cuda"), (3, 1, 515), (515, 7777, 1))
    z.copy_(i["z"])
    alike(want, losses.policy_loss(i["x"], i["y"], i["old"], i["adv"], ref_logits=z, kl_coef=0.1))


@pytest.mark.parametrize("native", [True, False])
def test_refusals(monkeypatch, native):
    if not native:
        monkeypatch.setattr(losses, "_calls", None)
    i = inputs()
    x, y, old, adv, ref = i["x"], i["y"], i["old"], i["adv"], i["ref"]
    stats = losses.token_logprobs(x, y, want_stats=True)["stats"]
    bad = [
        (ValueError, lambda: losses.token_logprobs(x, y[:, :5])),
        (ValueError, lambda: losses.token_logprobs(x, y, mask=i["mask"][:3])),
        (TypeError, lambda: losses.token_logprobs(x, y, mask=i["mask"].float())),
        (TypeError, lambda: losses.token_logprobs(x, y.float())),
        (TypeError, lambda: losses.token_logprobs(x.half(), y)),
        (ValueError, lambda: losses.token_logprobs(x[..., ::2], y)),
        (ValueError, lambda: losses.token_logprobs(x[:1].expand(4, 6, 1003), y)),
        (ValueError, lambda: losses.token_logprobs(x, y, workspace=torch.empty(1 << 20, dtype=torch.uint8))),
        (losses.SpecSteerError, lambda: losses.token_logprobs(x, y, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))),
        (losses.SpecSteerError, lambda: losses.token_logprobs(x, y, temperature=0.0)),
        (losses.SpecSteerError, lambda: losses.token_logprobs(x, y, temperature=math.nan)),
        (losses.SpecSteerError, lambda: losses.token_logprobs(x.transpose(0, 1), y.T)),
        (ValueError, lambda: losses.token_logprobs_grad(x, y, stats[:, :3], old)),
        (ValueError, lambda: losses.token_logprobs_grad(x, y, stats.double(), old)),
        (ValueError, lambda: losses.token_logprobs_grad(x, y, stats, old[:, 1:])),
        (ValueError, lambda: losses.token_logprobs_grad(x, y, stats, old, grad_logits=x.float())),
        (ValueError, lambda: losses.policy_loss(x, y, old, adv[:3])),
        (ValueError, lambda: losses.policy_loss(x, y, old, adv, ref_logits=i["z"][:, :5])),
        (ValueError, lambda: losses.policy_loss(x, y, old, adv, kl_coef=0.1)),
        (ValueError, lambda: losses.policy_loss(x, y, old, adv, ref_logits=i["z"], ref_logprobs=ref)),
        (ValueError, lambda: losses.policy_loss(x, y, old, adv, ref_logits=i["z"], grad_logits=i["z"])),
        (ValueError, lambda: losses.policy_loss(x[:, 1:], y[:, 1:].contiguous(), old[:, 1:].contiguous(), adv[:, 1:].contiguous(), grad_logits=x[:, :-1])),
        (ValueError, lambda: losses.policy_loss(x, y, old, adv, want_grad=False, grad_logits=torch.empty_like(x))),
        (losses.SpecSteerError, lambda: losses.policy_loss(x, y, old, adv, clip_low=1.5)),
        (losses.SpecSteerError, lambda: losses.policy_loss(x, y, old, adv, grad_scale=math.inf)),
        (TypeError, lambda: losses.policy_loss(x, y, old.long(), adv)),
        (ValueError, lambda: losses.preference_loss(x[:3], y[:3])),
        (ValueError, lambda: losses.preference_loss(x, y, ref_logprobs=ref[:2])),
        (losses.SpecSteerError, lambda: losses.preference_loss(x, y, label_smoothing=0.7)),
        (losses.SpecSteerError, lambda: losses.preference_loss(x, y, beta=math.inf)),
    ]
    for k, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {k} was not refused")
