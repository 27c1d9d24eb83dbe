"""Sums of attention weights: queries that saw nothing, requests of more queries than stated, and the native argument checks of one query a request."""
import numpy as np
import pytest
import torch

from paper_2404_09526_amd import binding as esp
from test_gpu_evict import check_weights, exact_weights, i32, offsets, weights_case
from test_gpu_q4_marshal import calls

pytestmark = pytest.mark.gpu

# heads and the queries of three requests, one for each kernel: one query a request (whole rows of four and eight heads where they are in 4 bits), several queries in one
# block of columns, many over short lists, many by tiles
QUERIES = [(8, 8, [1, 1, 1]), (8, 4, [1, 1, 1]), (6, 3, [5, 2, 4]), (8, 2, [30, 9, 3]), (40, 2, [2, 1, 3]), (4, 1, [19, 40, 2])]


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("hq,hkv,queries", QUERIES)
def test_a_query_that_saw_nothing_gives_nothing_whatever_it_holds(cuda, hq, hkv, queries, positions, bits):
    """Rows behind the last query of a padded batch: LSE = -inf, and q was never written."""
    c = weights_case(cuda, [300, 77, 131], queries, hq, hkv, bits, hq, positions)
    nothing = np.arange(sum(queries)) % 2 == 1
    c["LSE"][nothing] = -np.inf
    c["LSE"][0, hq // 2] = -np.inf                                    # and one head of a query
    c["q"][nothing] = 0
    c["q"][0, hq // 2] = 0
    c["q_dev"][torch.from_numpy(nothing).to(cuda)] = float("nan")
    c["q_dev"][0, hq // 2, ::2] = float("inf")
    check_weights(c, decay=0.5, by_offsets=True)


def first_queries(c, most):
    """The case with the first `most` queries of each request alone."""
    at = offsets(c["queries"])
    rows = np.concatenate([np.arange(at[b], at[b] + min(most, n)) for b, n in enumerate(c["queries"])]).astype(int)
    return dict(c, queries=np.minimum(c["queries"], most), q=c["q"][rows], LSE=c["LSE"][rows], q_pos=None if c["q_pos"] is None else c["q_pos"][rows])


@pytest.fixture(params=[False, True], ids=["", "validated"])
def validating(cuda, request):
    was = esp.esp_debug_set_validate(request.param)
    yield request.param
    esp.esp_debug_set_validate(was)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("hq,hkv,queries,most", [(4, 4, [3, 1, 2], 1), (8, 8, [3, 0, 2], 1), (6, 3, [5, 2, 4], 2), (8, 2, [30, 9, 3], 7), (40, 2, [2, 1, 3], 1), (4, 1, [19, 40, 2], 9)])
def test_of_more_queries_than_stated_the_first_count(cuda, validating, hq, hkv, queries, most, positions, bits):
    c = weights_case(cuda, [300, 77, 131], queries, hq, hkv, bits, hq, positions)
    args = dict(q=c["q_dev"], LSE=torch.from_numpy(c["LSE"]).to(cuda), k_pool=c["pool"], slot_idx=i32(c["slot"], cuda), seq_offsets=i32(offsets(c["lens"]), cuda), max_len=300,
                weight_sum=torch.from_numpy(c["sums"]).to(cuda), q_offsets=i32(offsets(queries), cuda), max_q=most, q_pos=None if c["q_pos"] is None else i32(c["q_pos"], cuda),
                kv_pos=None if c["kv_pos"] is None else i32(c["kv_pos"], cuda), decay=0.5, fresh=2)
    got = esp.esp_accumulate_attn_weights(**args).double().cpu().numpy()
    want, off = exact_weights(first_queries(c, most), 128 ** -0.5, 0.5, 2)
    assert (np.abs(got - want) <= off).all()
    if validating:                                                    # what the checks do refuse: offsets that decrease, or end elsewhere
        for at, x in ((1, offsets(queries)[2] + 1), (3, sum(queries) - 1), (0, 1)):
            bad = args["q_offsets"].clone()
            bad[at] = int(x)
            with pytest.raises(esp.EspError):
                esp.esp_accumulate_attn_weights(**dict(args, q_offsets=bad))


@pytest.mark.parametrize("name", ["weights", "weights_q4"])
def test_native_checks_take_one_query_a_request_by_name(cuda, monkeypatch, name):
    """max_q = 1 says what None does."""
    call, kw, _ = calls(esp, cuda)[name]
    taken, marshal = [], esp._marshal

    class Spy:
        def __getattr__(self, what):
            f = getattr(marshal, what)
            return lambda *a: (taken.append(f(*a)), taken[-1])[1]
    monkeypatch.setattr(esp, "_marshal", Spy())
    sums = []
    for max_q in (None, 1):
        kw["weight_sum"].fill_(1)
        sums.append(call(**(kw | dict(max_q=max_q))).clone())
    assert taken == [0, 0] and torch.equal(*sums)
    for bad in (0, 2, -1, 1 << 32):
        with pytest.raises((ValueError, esp.EspError)):
            call(**(kw | dict(max_q=bad)))
