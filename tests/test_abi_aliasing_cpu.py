"""Operands that a launch reads while it writes others may not share memory with them, except in place where the header
says so.  Host-side validation alone: the addresses are made up, and a call that passes this check is refused for them
afterwards."""
import random

import paper_2405_13954_amd as P
from test_abi_adapters_cpu import backward, forward

AT = 1 << 40   # an address that no check before the pointers' kinds looks at


def dropout(rows, cols, x, ld_x, out, ld_out, res=None, ld_res=0):
    return P.lib().logra_dropout(x, ld_x, 1, rows, cols, 0.1, 1, 2, res, ld_res, out, ld_out, None)


def loss(rows, vocab, z, ld, dz, ld_d):
    return P.lib().logra_token_loss(z, ld, 1, rows, vocab, None, None, None, dz, ld_d, None)


def refused(status):
    """Refused for sharing memory; refusals for other reasons are of what comes after."""
    assert status == P.ERR_INVALID_ARG
    return "share memory" in P.logra_last_error()


def test_dx_does_not_share_memory_with_x():
    # dA's workgroups read x in the launch whose others store dx
    L = P.lib()
    ends = dict(rows=4, n_in=64, x=AT, ld_x=64, dA=AT * 2, dB=AT * 2 + (1 << 20))
    assert refused(backward(L, **ends, dx=AT, ld_dx=64))
    assert refused(backward(L, **ends, dx=AT + 3 * 128 + 112, ld_dx=64))         # the last 16 bytes of x
    assert refused(backward(L, **ends, dx=AT - 3 * 128 - 112, ld_dx=64))
    assert refused(backward(L, **ends, dx=AT, ld_dx=128))
    assert not refused(backward(L, **ends, dx=AT + 4 * 128, ld_dx=64))           # the rows behind x
    assert not refused(backward(L, **ends, dx=AT - 4 * 128, ld_dx=64))
    assert not refused(backward(L, **{**ends, "ld_x": 128}, dx=AT + 128, ld_dx=128))   # the other half of a buffer
    assert not refused(backward(L, **ends))


def test_bases_are_in_place_or_apart():
    L = P.lib()
    for call, base, out, width, far in ((forward, "base", "y", 32, dict(x=AT * 2)),
                                        (backward, "base", "dx", 64, dict(x=AT * 2, dA=AT * 3, dB=AT * 4))):
        ld_b, ld_o = f"ld_{base}", f"ld_{out}"
        assert not refused(call(L, **far, **{base: AT, out: AT, ld_b: width, ld_o: width}))
        assert refused(call(L, **far, **{base: AT, out: AT, ld_b: width, ld_o: 2 * width}))
        assert refused(call(L, **far, **{base: AT, out: AT + 2 * width, ld_b: width, ld_o: width}))     # one row on
        assert refused(call(L, **far, **{base: AT + 16, out: AT, ld_b: 2 * width, ld_o: 2 * width}))
        assert not refused(call(L, **far, **{base: AT + 2 * width, out: AT, ld_b: 2 * width, ld_o: 2 * width}))


def test_dropout_and_loss_are_in_place_or_apart():
    assert not refused(dropout(9, 24, AT, 24, AT, 24)) and refused(dropout(9, 24, AT, 24, AT + 48, 24))
    assert not refused(dropout(9, 24, AT, 24, AT * 2, 24, AT * 2, 24))
    assert refused(dropout(9, 24, AT, 24, AT * 2, 24, AT * 2, 32)) and refused(dropout(9, 24, AT, 24, AT * 2, 24, AT * 2 + 16, 24))
    assert not refused(dropout(1, 24, AT, 24, AT, 32))                           # one row: no stride
    assert not refused(loss(5, 100, AT, 104, AT, 104)) and refused(loss(5, 100, AT, 104, AT, 112))
    assert refused(loss(5, 100, AT, 104, AT + 208, 104)) and not refused(loss(5, 100, AT, 208, AT + 208, 208))


def test_sharing_is_that_of_the_bytes():
    # every answer against the sets of bytes, with equal and unequal strides, widths that end inside a row's gap, and
    # starts of either order
    g = random.Random(4)
    seen = {True: 0, False: 0}
    for _ in range(3000):
        rows, cols = g.randint(1, 6), g.randint(1, 40)
        least = -(-cols // 8)
        ld_x = 8 * (least + g.choice((0, 0, 1, 3, 9)))
        ld_o = g.choice((ld_x, 8 * (least + g.randint(0, 9))))
        shift = 2 * g.randint(-3 * ld_x * rows, 3 * ld_x * rows)
        if shift == 0:
            continue
        x = {r * 2 * ld_x + b for r in range(rows) for b in range(2 * cols)}
        out = {shift + r * 2 * ld_o + b for r in range(rows) for b in range(2 * cols)}
        want = bool(x & out)
        assert refused(dropout(rows, cols, AT, ld_x, AT + shift, ld_o)) == want, (rows, cols, ld_x, ld_o, shift)
        seen[want] += 1
    assert min(seen.values()) > 500
