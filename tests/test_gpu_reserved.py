"""Reserved tokens stay open through calls that are refused or change no slot,
and are closed by those that do."""

import pytest

from paper_2602_22603_amd import workload as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sq():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2602_22603_amd import sq as sqmod
    sqmod.lib()
    return sqmod


def _store(sq):
    s = sq.Store(2, 8, 2, 64, num_pages=12, max_seqs=4, max_pages_per_seq=6)
    a, b = s.seq_create(), s.seq_create()
    k = wl.device_normal_bf16((2, 40, 2, 64), 1, "cuda")
    for h in (a, b):
        s.append(h, k, k)
        s.span_mark(h, 0, 3, 3)
        s.span_mark(h, 1, 4, 9)
    return s, a, b


def _layer(s, layer):
    x = [wl.device_normal_bf16((5, n, 64), n + layer, "cuda") for n in (8, 2, 2)]
    s.qkv_store(layer, *x)
    return x


# a call of (store, the reserved sequence, another one), and whether it is refused
KEPT = [
    (lambda s, a, b: s.evict(a, [7]), True), (lambda s, a, b: s.evict(b, [7]), True),
    (lambda s, a, b: s.evict(b, [1, 7], deferred=True), True), (lambda s, a, b: s.evict(b, []), False),
    (lambda s, a, b: s.evict(b, [0]), False), (lambda s, a, b: s.evict(b, [0], deferred=True), False),
    (lambda s, a, b: s.compact(a), False), (lambda s, a, b: s.span_mark(a, 5, 40, 45), False),
    (lambda s, a, b: s.truncate(a, 99), True), (lambda s, a, b: s.fork(b, 99), True),
    (lambda s, a, b: s.reserve([b], [0]), True), (lambda s, a, b: s.draft_begin([b], [[0]]), True),
    (lambda s, a, b: s.step_begin([a, a]), True), (lambda s, a, b: s.release(3), True)]


@pytest.mark.parametrize("call,refused", KEPT)
def test_open_tokens_stay_open(sq, call, refused):
    import torch
    s, a, b = _store(sq)
    s.reserve([a], [5])
    _layer(s, 0)
    if refused:
        with pytest.raises(sq.SqError):
            call(s, a, b)
    else:
        call(s, a, b)
    q, k, v = _layer(s, 1)
    page, slots = s.page_table(a)[2], slice(8, 13)
    assert torch.equal(s.k_pool[1, :, page, slots].transpose(0, 1), k)
    assert torch.equal(s.v_pool[1, :, page, :, slots].permute(2, 0, 1), v)


@pytest.mark.parametrize("call", [
    lambda s, a, b: s.evict(a, [1]), lambda s, a, b: s.evict(b, [1]), lambda s, a, b: s.evict(b, [1], deferred=True),
    lambda s, a, b: s.truncate(b, 30), lambda s, a, b: s.fork(b, 20), lambda s, a, b: s.release(b),
    lambda s, a, b: s.step_begin([b])])
def test_open_tokens_are_closed(sq, call):
    s, a, b = _store(sq)
    s.reserve([a], [5])
    _layer(s, 0)
    call(s, a, b)
    with pytest.raises(sq.SqError):
        _layer(s, 1)


def test_a_refused_eviction_still_ends_a_step(sq):
    s, a, b = _store(sq)
    x = [wl.device_normal_bf16((1, n, 64), n, "cuda") for n in (2, 2, 8)]
    s.step_begin([a])
    s.step_attn(0, *x)
    with pytest.raises(sq.SqError):
        s.evict(b, [7])
    with pytest.raises(sq.SqError):
        s.step_attn(1, *x)
