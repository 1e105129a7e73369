"""That the limits of tests/delta_norms.py let the right results through, rounded to their types, and no wrong ones (CPU)."""
import pytest
import torch

from tests import delta_norms as norms, delta_reference as ref

# T, N, H, Hk, dk, dv, type; the last one is long enough to be cut into pieces
CASES = [(64, 2, 2, 2, 64, 64, "fp32"), (64, 2, 2, 1, 64, 64, "bf16"), (20, 2, 2, 2, 128, 128, "fp32"), (70, 2, 2, 1, 128, 128, "bf16"),
         (333, 1, 2, 2, 32, 64, "fp32"), (1100, 1, 2, 1, 128, 128, "bf16")]
L = 17.0


def name_of(c):
    return "-".join(map(str, c))


@pytest.fixture(scope="module", params=CASES, ids=name_of)
def case(request):
    T, N, H, Hk, dk, dv, dtype = request.param
    x, do, ds = ref.make(T, N, H, Hk, dk, dv, dtype, seed=T + dk, p_done=0.01, device="cpu")
    x["done"][:] = 0
    if T > 40:
        x["done"][40, 0] = 1
    want, _ = ref.oracle(x)
    want.update(ref.oracle(x, None, do, ds)[0])
    narrow = ("o", "dq", "dk", "dv") if dtype == "bf16" else ()
    right = {n: y.to(torch.bfloat16 if n in narrow else torch.float32) for n, y in want.items()}
    return request.param, x, do, ds, want, right


def off(case, name, wrong):
    (T, N, H, Hk, dk, dv, dtype), want = case[0], case[4]
    return norms.over(name, wrong, want[name], dk, dv, L, dtype == "bf16", T)


def test_right_results_pass(case):
    for name, y in case[5].items():
        assert off(case, name, y) <= 1.0, name
        assert case[0][6] == "bf16" or off(case, name, y) <= 0.5, name  # (a single rounding is a small part of the limit)


def test_zeros_and_other_signs(case):
    for name, y in case[5].items():
        assert off(case, name, 0 * y) > 1.0 and off(case, name, -y) > 1.0, name


def test_one_head_of_one_row(case):
    for name, y in case[5].items():
        wrong = y.clone()
        (wrong if name in norms.BY_STATE else wrong.transpose(0, 1))[0].select(0 if name in norms.BY_STATE else 1, -1).zero_()
        assert off(case, name, wrong) > 1.0, name


def test_one_step_of_one_head(case):
    """As a decay's gradient was lost once, behind an episode's begin."""
    for name, y in case[5].items():
        if name in norms.BY_STATE:
            continue
        wrong = y.clone()
        wrong[11, 0, 0] = 0
        assert case[0][6] == "bf16" and name not in ("dlog_decay", "dbeta") or off(case, name, wrong) > 1.0, name


def test_another_rounding_to_bf16(case):
    for name, y in case[4].items():
        wrong = y.float().bfloat16()
        if case[5][name].dtype == torch.bfloat16:
            wrong = (wrong.float() * (1.0 + 2.0 ** -8.5)).bfloat16()
        assert off(case, name, wrong.float()) > 1.0, name


def test_a_state_that_loses_its_third_term(case):
    """Passed from chunk to chunk as two bf16 numbers."""
    (T, N, H, Hk, dk, dv, dtype), x = case[:2]

    def two(s):
        a = s.float()
        cut = lambda b: (b.view(torch.int32) & -65536).view(torch.float32)
        return cut(a) + cut(a - cut(a))

    s = x["state0"]
    for t in range(0, T, 32):
        s = ref.oracle(dict({n: a[t:t + 32] for n, a in x.items() if n != "state0"}, state0=two(s)))[0]["state"]
    assert off(case, "state", two(s)) > 1.0


def test_a_chunk_without_what_both_its_states_give_its_decays(case):
    """What the state that enters and the gradient of the one behind give together: dlog_decay without it in the first chunk."""
    (T, N, H, Hk, dk, dv, dtype), x, do, ds = case[:4]
    cut = min(T, 32)
    first = {n: a[:cut] for n, a in x.items() if n != "state0"}
    behind = ds
    if T > cut:
        state = ref.oracle(dict(first, state0=x["state0"]))[0]["state"]
        behind = ref.oracle(dict({n: a[cut:] for n, a in x.items() if n != "state0"}, state0=state), None, do[cut:], ds)[0]["dstate0"]
    f = lambda s, r: ref.oracle(dict(first, state0=s), None, do[:cut], r)[0]["dlog_decay"]
    both = f(x["state0"], behind) - f(x["state0"], None) - f(None, behind) + f(None, None)
    wrong = case[4]["dlog_decay"].clone()
    wrong[:cut] -= both
    assert off(case, "dlog_decay", wrong) > 1.0
