"""CPU tests of the 64-bit definitions that the output head's kernels are held to:
hand-written values, gradients against differences, and the arguments the C ABI
refuses before any device work."""
import ctypes
import math

import numpy as np
import pytest

from tests import head_oracle as O

INF = math.inf


def test_hand_written_rows():
    lp, H, (m, log_s), ids, tl = O.token_logprobs([0.0, math.log(3.0)], 0, 1.0, 2)
    assert lp == pytest.approx(math.log(0.25)) and m == math.log(3.0)
    assert H == pytest.approx(-(0.25 * math.log(0.25) + 0.75 * math.log(0.75)))
    assert list(ids) == [1, 0] and tl[1] == pytest.approx(lp)
    lp, H, st, ids, tl = O.token_logprobs([-INF, -INF, -INF], 1, 1.0, 2)
    assert (lp, H, st, list(ids), list(tl)) == (-INF, 0.0, (-INF, 0.0), [0, 1], [-INF, -INF])
    lp, H, _, ids, _ = O.token_logprobs([1.0, -INF, 1.0, -0.0, 0.0], 0, 1.0, 4)
    assert list(ids) == [0, 2, 3, 4]
    low = -3.3895313892515355e38
    lp, H, _, _, _ = O.token_logprobs([low] * 8, 3, 2.0, 0)
    assert lp == pytest.approx(-math.log(8)) and H == pytest.approx(math.log(8))
    # a list that is all there is: KL of two distributions
    loss, _ = O.distill([0.0, 0.0], [0, 1], [math.log(3.0), 0.0], 1.0, False)
    assert loss == pytest.approx(0.75 * math.log(1.5) + 0.25 * math.log(0.5))
    # the rest class: q = (1/2, rest 1/2), p = (1/4, rest 3/4)
    loss, g = O.distill([0.0] * 4, [2], [math.log(0.5)], 1.0, True)
    assert loss == pytest.approx(0.5 * math.log(2) + 0.5 * math.log(0.5 / 0.75))
    assert g == pytest.approx([0.25 - 0.5 / 3, 0.25 - 0.5 / 3, 0.25 - 0.5, 0.25 - 0.5 / 3])


def _differences(f, x, h=1e-5):
    g = np.zeros(len(x))
    for v in range(len(x)):
        a, b = x.copy(), x.copy()
        a[v] += h
        b[v] -= h
        g[v] = (f(a) - f(b)) / (2 * h)
    return g


@pytest.mark.parametrize("scale", [1.0, 0.6])
def test_gradients_are_the_differences(scale):
    rng = np.random.default_rng(1)
    x = rng.normal(size=11) * 2

    def combined(y):
        lp, H, (m, log_s), _, _ = O.token_logprobs(y, 4, scale)
        return 0.7 * lp - 1.3 * H + 0.4 * (scale * m + log_s)

    assert np.allclose(O.token_logprobs_grad(x, 4, scale, 0.7, -1.3, 0.4), _differences(combined, x),
                       atol=1e-8)
    ids = np.array([3, -1, 7, 3, 0])          # one id twice, one entry absent
    values = np.log(np.array([0.2, 0.9, 0.3, 0.1, 0.05]))
    for rest in (False, True):
        f = lambda y: O.distill(y, ids, values, scale, rest)[0]  # noqa: E731
        assert np.allclose(O.distill(x, ids, values, scale, rest)[1], _differences(f, x), atol=1e-8)


def _status(name, *args):
    import paper_2511_12500_amd as pkg
    with pytest.raises(pkg.SymtileError) as e:
        getattr(pkg, name)(*args)
    return e.value.name, str(e.value)


P = 1 << 20      # an aligned address that is never read: the calls below are refused


@pytest.mark.parametrize("change,word", [
    (dict(dtype=9), "dtype"), (dict(rows=-1), "rows"), (dict(vocab=0), "vocab"),
    (dict(ld=99), "ld"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"),
    (dict(scale=INF), "scale"), (dict(scale=math.nan), "scale"), (dict(logits=0), "NULL"),
    (dict(logits=P + 1), "aligned"), (dict(targets=0), "together"), (dict(logprob=0), "together"),
    (dict(top=129), "top"), (dict(top=-1), "top"), (dict(vocab=4, top=5), "top"),
    (dict(top=2, top_ids=0), "top"), (dict(top=2, top_logprobs=0), "top"),
    (dict(grad_lse=P), "without dlogits"), (dict(dlogits=P + 64), "overlaps"),
    (dict(dlogits=P, ld_grad=200), "overlaps"), (dict(dlogits=P + 4096, ld_grad=99), "ld_grad"),
    (dict(dlogits=P + 8193), "aligned"), (dict(dlogits=P + 8192, stats=0), "stats"),
    (dict(dlogits=P + 8192, entropy=0), "entropy"),
    (dict(dlogits=P + 8192, targets=0, logprob=0, grad_logprob=P), "targets"),
])
def test_token_logprobs_refuses(change, word):
    a = dict(device=0, logits=P, rows=4, vocab=100, ld=100, dtype=2, scale=1.0, targets=P,
             logprob=P, entropy=P, stats=P, top=0, top_ids=P, top_logprobs=P, grad_logprob=0,
             grad_entropy=0, grad_lse=0, dlogits=0, ld_grad=0)
    a.update(change)
    name, text = _status("symtile_token_logprobs", *a.values())
    assert name == "EINVAL" and word in text, text


@pytest.mark.parametrize("change,word", [
    (dict(k=0), "k must"), (dict(k=129), "k must"), (dict(values_dtype=0), "values_dtype"),
    (dict(mode=2), "mode"), (dict(ids=0), "NULL"), (dict(values=0), "NULL"),
    (dict(ids=P + 4), "aligned"), (dict(values=P + 2), "aligned"), (dict(loss=0), "loss"),
    (dict(row_grad=P), "without dlogits"), (dict(dlogits=P + 8192), "row_grad"),
    (dict(dlogits=P + 8192, row_grad=P, stats=0), "stats"), (dict(dlogits=P + 32, row_grad=P), "overlaps"),
    (dict(dtype=0), "dtype"), (dict(ld=50), "ld"),
])
def test_distill_refuses(change, word):
    a = dict(device=0, logits=P, rows=4, vocab=100, ld=100, dtype=1, scale=1.0, ids=P, values=P,
             values_dtype=3, k=5, mode=0, loss=P, stats=P, row_grad=0, dlogits=0, ld_grad=0)
    a.update(change)
    name, text = _status("symtile_distill_topk", *a.values())
    assert name == "EINVAL" and word in text, text


def test_backward_calls_refuse():
    base = (0, P, 4, 100, 100, 2, 1.0)
    assert "dlogits" in _status("symtile_token_logprobs_backward", *base, P, P, P, P, 0, 0, 0)[1]
    assert "stats" in _status("symtile_token_logprobs_backward", *base, P, P, 0, P, 0, 0, P + 8192)[1]
    assert "targets" in _status("symtile_token_logprobs_backward", *base, 0, P, P, P, 0, 0, P + 8192)[1]
    assert "row_grad" in _status("symtile_distill_topk_backward", *base, P, P, 3, 5, 0, P, 0, P + 8192)[1]
    assert "dlogits" in _status("symtile_distill_topk_backward", *base, P, P, 3, 5, 0, P, P, 0)[1]


def test_workspace_query_refuses():
    import paper_2511_12500_amd as pkg
    for bad in ((0, -1, 10, 2, 0), (0, 1, 0, 2, 0), (0, 1, 10, 7, 0), (0, 1, 10, 2, 11),
                (0, 1, 1000, 2, 129)):
        with pytest.raises(pkg.SymtileError) as e:
            pkg.symtile_logits_workspace_bytes(*bad)
        assert e.value.name == "EINVAL", bad
    assert pkg.lib.symtile_logits_workspace_bytes(0, 1, 10, 2, 0, None) == -1


def test_w4_without_a_heap_is_refused():
    import paper_2511_12500_amd as pkg
    assert pkg.lib.symtile_w4_all_scatter(None, P, P, P, None, P, P, 1, 16, 32, 0, 32, 2, 0, 1,
                                          None, 0, None) == -1
    assert b"NULL" in ctypes.string_at(pkg.lib.symtile_last_error())


def test_empty_calls_need_no_device_memory():
    """rows = 0 launches nothing and reads no pointer."""
    import paper_2511_12500_amd as pkg
    pkg.symtile_token_logprobs(0, 0, 0, 100, 0, 2, 1.0, 0, 0, 0, 0)
    pkg.symtile_distill_topk(0, 0, 0, 100, 0, 2, 1.0, 0, 0, 3, 5, 0, 0)
