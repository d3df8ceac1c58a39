"""The training-stage entry points on the CPU: struct layouts, enums, workspace
sizes and refusals.  No call here reaches the GPU."""
import ctypes as C
import re

import pytest
import torch

from paper_2509_15965_amd import rl_decode as R
from test_abi_host import HEADER, _compile_and_run

P = 4096           # a pointer that no refused call follows
WS = 1 << 40


def test_structs_and_enums_match_the_header(tmp_path):
    structs = {"rl_policy_params": R.PolicyParams, "rl_policy_batch": R.PolicyBatch,
               "rl_preference_params": R.PreferenceParams}
    body = ""
    for name, py in structs.items():
        body += f'printf("{name}=%zu\\n", sizeof({name}));\n'
        for f, _ in py._fields_:
            body += f'printf("{name}.{f}=%zu\\n", offsetof({name}, {f}));\n'
    enums = {"RL_KL_" + k.upper(): v for k, v in R.KL_KINDS.items()}
    enums |= {"RL_AGG_" + k.upper(): v for k, v in R.AGGREGATES.items()}
    enums |= {"RL_PREF_" + k.upper(): v for k, v in R.PREFERENCE_FORMS.items()}
    assert sorted(enums) == sorted(re.findall(r"\b(RL_(?:KL|AGG|PREF)_[A-Z0-9_]+)\s*=", open(HEADER).read()))
    body += "".join(f'printf("{k}=%d\\n", (int){k});\n' for k in enums)
    got = _compile_and_run(tmp_path, body)
    for name, py in structs.items():
        assert int(got[name]) == C.sizeof(py)
        for f, _ in py._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(py, f).offset, (name, f)
    for k, v in enums.items():
        assert int(got[k]) == v, k


def test_workspace_bytes():
    L = R.lib()
    for n, v in ((0, 8), (-1, 8), (1, 0), (1, (1 << 24) + 1), ((1 << 20) + 1, 8)):
        assert L.rl_logprob_workspace_bytes(n, v) == 0
        if n:
            assert L.rl_policy_logits_workspace_bytes(n, 1, v) == 0
    assert L.rl_logprob_workspace_bytes(1, 152064) > 0            # one row is cut
    assert L.rl_logprob_workspace_bytes(1 << 20, 1000) == 0
    for n, k in ((-1, 1), (1, 0), ((1 << 24) + 1, 1), (1, (1 << 20) + 1)):
        assert L.rl_policy_workspace_bytes(n, k) == 0
    for n, k in ((-1, 1), (1, 0), ((1 << 24) + 1, 1), (1, (1 << 19) + 1)):
        assert L.rl_preference_workspace_bytes(n, k) == 0
    for n in (0, 1, 7, 1 << 20):
        assert L.rl_policy_workspace_bytes(n, 3) % 256 == 0
        assert L.rl_policy_logits_workspace_bytes(n, 3, 1000) % 256 == 0


def logprobs(n=2, vocab=100, dtype=1, logits=P, ld=100, targets=P, T=1.0, logp=P, ws=P, nb=WS):
    return R.lib().rl_token_logprobs(n, vocab, dtype, logits, ld, targets, T, logp, None, None, ws, nb, None)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=(1 << 20) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1, ld=1 << 25),
                                 dict(dtype=2), dict(dtype=-1), dict(ld=99), dict(ld=1 << 40), dict(logits=None),
                                 dict(logits=P + 1), dict(dtype=0, logits=P + 2), dict(targets=None), dict(logp=None),
                                 dict(T=-0.5), dict(T=float("nan")), dict(T=float("inf")),
                                 dict(n=1, vocab=152064, ld=152064, ws=None),
                                 dict(n=1, vocab=152064, ld=152064, ws=P + 16)])
def test_token_logprobs_refuses(bad):
    assert logprobs(**bad) == R.RL_ERR_INVALID_ARG


def test_token_logprobs_small_workspace_and_no_rows():
    assert logprobs(n=1, vocab=152064, ld=152064, nb=64) == R.RL_ERR_CAPACITY
    assert logprobs(n=0, logits=None, targets=None, logp=None) == R.RL_OK


def backward(n=2, vocab=100, dtype=1, logits=P, ld=100, targets=P, T=1.0, stats=P, ent=P, g=P, ge=P, dz=P, ldd=100):
    return R.lib().rl_token_logprobs_backward(n, vocab, dtype, logits, ld, targets, T, stats, ent, g, ge, dz, ldd, None)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(vocab=0), dict(dtype=3), dict(ldd=99), dict(logits=None), dict(targets=None),
                                 dict(stats=None), dict(g=None), dict(dz=None), dict(ent=None), dict(dz=P + 1),
                                 dict(T=float("nan")),
                                 dict(ldd=101),                        # in place, but rows elsewhere
                                 dict(dz=P + 2), dict(dz=P + 398),     # inside the logits
                                 dict(dz=P - 2), dict(ld=200, dz=P + 200)])
def test_backward_refuses(bad):
    assert backward(**bad) == R.RL_ERR_INVALID_ARG


def test_backward_no_rows():
    assert backward(n=0, logits=None, targets=None, stats=None, g=None, dz=None) == R.RL_OK


def policy(batch=(), params=(), logp=P, ent=P, out=P, g=P, ge=P, ws=P, nb=WS, logits=None):
    b = R.PolicyBatch(10000, 2, P, P, P, P, P)
    q = R.PolicyParams(0.2, 0.2, 0.0, 0.1, 0.01, 1.0, 3, 0, 0, 0)
    for k, v in dict(batch).items():
        setattr(b, k, v)
    for k, v in dict(params).items():
        setattr(q, k, v)
    if logits is not None:
        a = dict(vocab=100, dtype=1, z=P, ld=100, y=P, T=1.0, out=out, lp=P, ent=ent, dz=P, ldd=100) | logits
        return R.lib().rl_policy_loss_logits(C.byref(b), C.byref(q), a["vocab"], a["dtype"], a["z"], a["ld"], a["y"], a["T"],
                                             a["out"], a["lp"], a["ent"], a["dz"], a["ldd"], ws, nb, None)
    return R.lib().rl_policy_loss(C.byref(b), C.byref(q), logp, ent, out, g, ge, ws, nb, None)


NAN, INF = float("nan"), float("inf")
BAD_POLICY = [dict(batch=dict(n=-1)), dict(batch=dict(n=(1 << 24) + 1)), dict(batch=dict(n_seqs=0)),
              dict(batch=dict(n_seqs=(1 << 20) + 1)), dict(batch=dict(seq_offsets=None)), dict(batch=dict(old_logp=None)),
              dict(batch=dict(advantages=None)), dict(batch=dict(ref_logp=None)),
              dict(params=dict(clip_low=-0.1)), dict(params=dict(clip_low=1.0)), dict(params=dict(clip_low=NAN)),
              dict(params=dict(clip_high=-0.1)), dict(params=dict(clip_high=INF)), dict(params=dict(dual_clip=1.0)),
              dict(params=dict(dual_clip=-3.0)), dict(params=dict(dual_clip=INF)), dict(params=dict(kl_coef=NAN)),
              dict(params=dict(entropy_coef=INF)), dict(params=dict(scale=NAN)), dict(params=dict(kl=0)),
              dict(params=dict(kl=4)), dict(params=dict(aggregate=-1)), dict(params=dict(aggregate=3)),
              dict(params=dict(token_advantages=2)), dict(params=dict(reserved=1)), dict(out=None), dict(ws=None),
              dict(ws=P + 8), dict(ent=None)]


@pytest.mark.parametrize("bad", BAD_POLICY + [dict(logp=None), dict(g=None)])
def test_policy_loss_refuses(bad):
    assert policy(**bad) == R.RL_ERR_INVALID_ARG


def test_policy_null_structs_and_small_workspace():
    L = R.lib()
    q = R.PolicyParams(0.2, 0.2, 0.0, 0.0, 0.0, 1.0, 3, 0, 0, 0)
    b = R.PolicyBatch(10, 2, P, P, P, P, P)
    assert L.rl_policy_loss(None, C.byref(q), P, P, P, P, P, P, WS, None) == R.RL_ERR_INVALID_ARG
    assert L.rl_policy_loss(C.byref(b), None, P, P, P, P, P, P, WS, None) == R.RL_ERR_INVALID_ARG
    assert policy(nb=8) == R.RL_ERR_CAPACITY
    assert policy(nb=8, logits={}) == R.RL_ERR_CAPACITY


@pytest.mark.parametrize("bad", BAD_POLICY + [dict(logits=k) for k in (
    dict(vocab=0), dict(dtype=2), dict(z=None), dict(z=P + 1), dict(ld=99), dict(y=None), dict(T=-1.0), dict(lp=None),
    dict(dz=None), dict(dz=P + 2), dict(ldd=99), dict(ldd=101), dict(ent=None))])
def test_policy_loss_logits_refuses(bad):
    if bad.get("batch") == dict(n=(1 << 24) + 1):
        bad = dict(batch=dict(n=(1 << 20) + 1))
    assert policy(**(dict(logits={}) | bad)) == R.RL_ERR_INVALID_ARG


def preference(n=100000, pairs=2, offs=P, logp=P, params=(), out=P, g=P, ws=P, nb=WS):
    q = R.PreferenceParams(0.1, 0.0, 0.0, 1.0, 0, 0)
    for k, v in dict(params).items():
        setattr(q, k, v)
    return R.lib().rl_preference_loss(n, pairs, offs, logp, P, P, C.byref(q), out, P, g, ws, nb, None)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=(1 << 24) + 1), dict(pairs=0), dict(pairs=(1 << 19) + 1), dict(offs=None),
                                 dict(logp=None), dict(out=None), dict(g=None), dict(ws=None), dict(ws=P + 8),
                                 dict(params=dict(beta=0.0)), dict(params=dict(beta=NAN)), dict(params=dict(beta=INF)),
                                 dict(params=dict(label_smoothing=-0.1)), dict(params=dict(label_smoothing=0.6)),
                                 dict(params=dict(form=1, label_smoothing=0.1)), dict(params=dict(margin=NAN)),
                                 dict(params=dict(scale=INF)), dict(params=dict(form=3)), dict(params=dict(form=-1)),
                                 dict(params=dict(average=2))])
def test_preference_loss_refuses(bad):
    assert preference(**bad) == R.RL_ERR_INVALID_ARG


def test_preference_small_workspace():
    assert preference(nb=8) == R.RL_ERR_CAPACITY


def test_binding_refuses_host_tensors():
    z, y, f = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    with pytest.raises(ValueError, match="GPU"):
        R.token_logprobs(z, y, f)
    with pytest.raises(ValueError, match="GPU"):
        R.token_logprobs_backward(z, y, torch.zeros(2, 2), f, z)
    with pytest.raises(ValueError, match="GPU"):
        R.policy_loss(f, f, f, torch.zeros(8), f)
    with pytest.raises(ValueError, match="GPU"):
        R.policy_loss_logits(z, y, f, f, torch.zeros(8), f, z)
    with pytest.raises(ValueError, match="GPU"):
        R.preference_loss(f, torch.zeros(3, dtype=torch.int32), torch.zeros(8), f)


@pytest.mark.parametrize("T", [1e-31, 1e-300, 2e30, 1e300, -0.0])
def test_temperatures_out_of_range(T):
    # -0.0 is 0: taken as 1 (no rows, so nothing runs)
    want = R.RL_OK if T == 0 else R.RL_ERR_INVALID_ARG
    assert logprobs(n=0, T=T) == want and backward(n=0, T=T) == want
    if T:
        assert policy(logits=dict(T=T)) == want


def test_interleaved_gradient_rows_are_refused():
    # d_logits' rows between the logits' rows: neither in place nor apart
    assert backward(ld=200, ldd=200, dz=P + 200) == R.RL_ERR_INVALID_ARG
    assert policy(logits=dict(ld=200, ldd=200, dz=P + 200)) == R.RL_ERR_INVALID_ARG
