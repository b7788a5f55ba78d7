"""What the marshalling helpers of the logit rules and the optimizer table refuse: tensors that a call would read past the end of,
or could not read at all."""
import gc
import weakref

import pytest
import torch

from paper_2609_33570_b200 import api, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return api.lib()


def rows_of(n):
    i = lambda k=n: torch.zeros(k, dtype=torch.int64)
    return dict(temperature=torch.ones(n), repetition=torch.ones(n), frequency=torch.zeros(n), presence=torch.zeros(n),
                tokens=torch.zeros(9, dtype=torch.int32), hist_begin=i(), resp_begin=i(), hist_end=i(), bias_offsets=i(n + 1),
                bias_tokens=torch.zeros(5, dtype=torch.int32), bias_values=torch.zeros(5), allow=torch.zeros(2, 4, dtype=torch.int32),
                allow_row=torch.zeros(n, dtype=torch.int32))


@pytest.mark.parametrize("name", ["temperature", "repetition", "frequency", "presence", "hist_begin", "resp_begin", "hist_end", "bias_offsets",
                                  "allow_row"])
def test_rules_have_the_rows_of_their_shortest_part(name):
    good = rows_of(4)
    assert api.make_logit_rules(**good).rows == 4
    assert api.make_logit_rules(**dict(good, **{name: good[name][:-1]})).rows == 3
    assert api.make_logit_rules(**dict(good, **{name: torch.cat([good[name], good[name][:1]])})).rows == 4


def test_rules_of_other_shapes():
    good = rows_of(4)
    with pytest.raises(ValueError, match="4 bias_values of 5"):
        api.make_logit_rules(**dict(good, bias_values=torch.zeros(4)))
    with pytest.raises(ValueError, match="allow: expected"):
        api.make_logit_rules(**dict(good, allow=torch.zeros(8, dtype=torch.int32)))
    assert api.make_logit_rules().rows is None and not api.make_logit_rules().on_host


def test_parts_that_no_call_reads_ask_for_nothing():
    some = {k: v for k, v in rows_of(4).items() if k not in ("tokens", "bias_tokens", "allow", "temperature")}
    r = api.make_logit_rules(**dict(some, temperature=torch.ones(9)))
    assert r.rows == 4 and set(r.on_host) == {"temperature", "repetition", "frequency", "presence"}
    few = dict(hist_begin=torch.zeros(1, dtype=torch.int64), bias_offsets=torch.zeros(1, dtype=torch.int64), allow_row=torch.zeros(1, dtype=torch.int32))
    r = api.make_logit_rules(**few)
    assert r.rows is None and r.on_host == ()


def test_calls_of_more_rows_than_the_rules_have(lib):
    a = 0x1000  # a fake device address: refused before it is read
    short = api.make_logit_rules(temperature=torch.ones(3))
    for call in (lambda n: api.hilore_logits_apply(a, api.F32, n, 8, 8, short, a, 8, stream=0),
                 lambda n: api.hilore_logits_apply_backward(a, api.F32, n, 8, 8, short, 2 * a, 8, 3 * a, 8, stream=0),
                 lambda n: api.hilore_token_logp(a, api.F32, n, 8, 8, short, a, a, None, None, stream=0),
                 lambda n: api.hilore_token_logp_backward(a, api.F32, n, 8, 8, short, a, a, a, a, 8, stream=0)):
        with pytest.raises(ValueError, match="3 rows in a call of 4"):
            call(4)
        with pytest.raises(ValueError, match="temperature: expected device tensors"):
            call(3)
        with pytest.raises(ValueError, match="temperature: expected device tensors"):
            call(2)


def entry(n=130):
    return dict(p=torch.zeros(n), g=torch.zeros(n), m=torch.zeros(n), v=torch.zeros(n))


def test_tables_of_host_tensors_and_of_fewer_entries(lib):
    with pytest.raises(ValueError, match="entry 0: p is on the host, the table on cuda"):
        api.make_param_table([entry()])
    _, host = api.make_param_table([entry(), entry()], device="cpu")
    a = 0x1000
    with pytest.raises(ValueError, match="2 entries in a call of 3"):
        api.hilore_adamw_step(a, host, 3, 1e-3, None, 0.9, 0.99, 1e-8, 1, None, None, stream=0)
    with pytest.raises(ValueError, match="2 entries in a call of 3"):
        api.hilore_grad_norm(a, host, 3, 1.0, a, None, a, 1 << 20, stream=0)


def test_a_table_keeps_its_tensors_when_the_caller_lets_go():
    entries = [entry()]
    alive = weakref.ref(entries[0]["m"])
    _, host = api.make_param_table(entries, device="cpu")
    entries[0].clear()
    entries.clear()
    gc.collect()
    assert alive() is not None
    del host
    gc.collect()
    assert alive() is None
