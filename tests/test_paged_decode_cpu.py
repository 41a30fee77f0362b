"""CPU: how pipeline.PagedDecode counts tokens: what is not there, has no room or no pages does not grow, and a token sees its own sequence's
slots and nothing else."""
import pytest
import torch

from tests.paged_fakes import INVALID, OK, decode, keep, step


def test_places_without_a_sequence_do_not_grow(monkeypatch):
    """One sequence decodes, then others begin in places that had none, or whose sequence had ended."""
    dec = decode(monkeypatch, pages=12, columns=4, batch=3)
    dec.reserve(0, 40)
    keep(dec, 0, 30)
    for _ in range(5):
        step(dec)
        dec.advance(1)
    assert dec.lengths.tolist() == [35, 0, 0]
    dec.reserve(1, 40)
    keep(dec, 1, 20)
    dec.release(0)
    dec.advance(1)
    assert dec.lengths.tolist() == [0, 21, 0]
    dec.reserve(0, 40)
    keep(dec, 0, 10)
    dec.ctx.poll_device_status()
    seen = step(dec, counts=torch.tensor([1, 1, 0], dtype=torch.int32))
    assert seen[0] == [0] * 11 and len(seen[1]) == 22 and dec.ctx.poll_device_status() == OK
    dec.reserve(2, 1)
    assert dec.lengths.tolist() == [10, 21, 0]


def test_a_full_sequence_stays_as_it_is(monkeypatch):
    """No slot is left for a token: its length stays, the status word says so, and a token that fits goes on from there."""
    dec = decode(monkeypatch, pages=8, columns=2, batch=2)
    dec.reserve(0, 32)
    dec.reserve(1, 32)
    keep(dec, 0, 31)
    keep(dec, 1, 5)
    assert dec.ctx.poll_device_status() == OK
    step(dec, 2)
    assert dec.ctx.poll_device_status() == INVALID
    dec.advance(2)
    assert dec.lengths.tolist() == [31, 7] and dec.ctx.poll_device_status() == INVALID
    seen = step(dec)
    dec.advance(1)
    assert [len(x) for x in seen] == [32, 8] and dec.lengths.tolist() == [32, 8] and dec.ctx.poll_device_status() == OK


def test_tokens_without_a_page_do_not_count(monkeypatch):
    """The next page was not reserved: nothing was written there, so that nothing of it counts once the page is there, whoever had it before."""
    dec = decode(monkeypatch, pages=2, columns=2, batch=2)
    dec.reserve(1, 16)
    keep(dec, 1, 16)
    dec.reserve(0, 16)
    keep(dec, 0, 15)
    for _ in range(3):
        step(dec)
        dec.advance(torch.tensor([1, 0], dtype=torch.int32))
    assert dec.lengths.tolist() == [16, 16] and dec.ctx.poll_device_status() == INVALID
    dec.release(1)
    dec.reserve(0, 20)
    seen = step(dec, counts=torch.tensor([1, 0], dtype=torch.int32))
    assert seen[0] == [0] * 17 and dec.ctx.poll_device_status() == OK


def test_counts_that_cannot_be(monkeypatch):
    dec = decode(monkeypatch, pages=8, columns=2, batch=4)
    for b in range(3):
        dec.reserve(b, 20)
        keep(dec, b, 10)
    assert dec.ctx.poll_device_status() == OK
    dec.advance(torch.tensor([-11, 23, 22, 0], dtype=torch.int32))
    assert dec.lengths.tolist() == [10, 10, 32, 0] and dec.ctx.poll_device_status() == INVALID
    # a number of its own for a place without a sequence is a mistake; one number for all is not
    dec.advance(torch.tensor([1, 0, 0, 1], dtype=torch.int32))
    assert dec.lengths.tolist() == [11, 10, 32, 0] and dec.ctx.poll_device_status() == INVALID
    dec.release(2)
    dec.advance(2)
    assert dec.lengths.tolist() == [13, 12, 0, 0] and dec.ctx.poll_device_status() == OK


def test_a_batch_that_is_not_full_is_no_mistake(monkeypatch):
    """Places without a sequence have no new tokens: nothing is reported for them, step after step, and a real mistake can be told."""
    dec = decode(monkeypatch, pages=12, columns=4, batch=5)
    dec.reserve(1, 40)
    keep(dec, 1, 30)
    for n in (1, 4, 2):
        seen = step(dec, n)
        assert [len(x) for x in seen] == [0, int(dec.lengths[1]) + n, 0, 0, 0] and dec.ctx.poll_device_status() == OK
        dec.advance(1)
    dec.reserve(4, 16)
    assert [len(x) for x in step(dec, 3)] == [0, 36, 0, 0, 3] and dec.ctx.poll_device_status() == OK
    # ends, and begins anew
    dec.release(1)
    assert [len(x) for x in step(dec, 3)] == [0, 0, 0, 0, 3] and dec.ctx.poll_device_status() == OK
    dec.reserve(1, 2)
    assert [len(x) for x in step(dec, 3)] == [0, 3, 0, 0, 3] and dec.ctx.poll_device_status() == OK
    # counts of the caller's are taken as they are
    step(dec, 3, counts=torch.tensor([1, 1, 0, 0, 1], dtype=torch.int32))
    assert dec.ctx.poll_device_status() == INVALID


def test_positions_without_a_rope_are_refused(monkeypatch):
    """keep() would store K as it is where its caller expects it to be rotated."""
    dec = decode(monkeypatch, pages=4, columns=2, batch=1)
    dec.reserve(0, 20)
    k, v = (torch.zeros((2, 10, 64), dtype=torch.bfloat16) for _ in range(2))
    with pytest.raises(ValueError):
        dec.keep(0, 0, k, v, positions=torch.arange(10, dtype=torch.int32))
    dec.keep(0, 0, k, v)
