"""Views of one buffer in a call: refused where they share an element, taken where they do not.

No GPU: every call here lacks a pointer that is checked right after the views, so one whose
views are taken ends at that check."""
import random

import pytest

import paper_2604_20819_amd as cq
from tests.test_operator_args import PTR, cache, view


def attend(q, o):
    return cq.lib().cqsa_cache_attend(cache(H=1, d=q.d), cq.cqsa_cache_batch(PTR, 5, None, None, q.B, 5, 300, 0), q, o,
                                      None, 1, 0.0, None, 0, None)


def read(k, v):
    return cq.lib().cqsa_cache_read(cache(H=k.H, d=k.d), cq.cqsa_cache_batch(PTR, 5, None, None, k.B, 5, 300, 0), k, v, None)


def rotary(xs, ys):
    plan = cq.cqsa_rotary_plan(xs[0].d)
    a, b = ((cq.cqsa_view * 2)(*(list(t) * 2)[:2]) for t in (xs, ys))
    return cq.lib().cqsa_rotary(plan.handle, None, a, b, len(xs), 0, None)


def why(status):
    """Whether the call ended at its views ("shared") or behind them ("taken")."""
    assert status == -1
    text = cq.lib().cqsa_last_error().decode()
    if "lengths is NULL" in text or "pos is NULL" in text:
        return "taken"
    assert "overlap" in text or "one tensor" in text or "share" in text, text
    return "shared"


def part(first, heads, of=12, B=2, L=5, d=64, shift=0):
    """Heads first ... first + heads - 1 of a buffer [B, L, of, d] in bf16."""
    return view(B=B, L=L, H=heads, d=d, data=PTR + 2 * d * first + shift, stride_b=L * of * d, stride_l=of * d, stride_h=d)


def test_parts_of_one_projection():
    q = part(0, 4)
    assert why(attend(q, q)) == "taken"  # O is Q
    assert why(attend(q, part(4, 4))) == "taken"
    assert why(attend(q, part(8, 4))) == "taken"
    assert why(attend(q, part(1, 4))) == "shared"
    assert why(attend(part(3, 4), q)) == "shared"
    assert why(attend(q, part(4, 4, shift=-16))) == "shared"
    assert why(read(part(4, 2), part(6, 2))) == "taken"
    assert why(read(part(4, 2), part(5, 2))) == "shared"
    assert why(read(part(5, 2), part(4, 2))) == "shared"
    assert why(rotary([q], [q])) == "taken"
    assert why(rotary([q], [part(4, 4)])) == "taken"
    assert why(rotary([q], [part(3, 4)])) == "shared"
    k = part(4, 2)
    assert why(rotary([q, k], [q, k])) == "taken"
    assert why(rotary([q, k], [part(6, 4), part(10, 2)])) == "taken"
    assert why(rotary([q, k], [part(6, 4), part(9, 2)])) == "shared"   # the results share a head
    assert why(rotary([q, k], [part(5, 4), part(10, 2)])) == "shared"  # q's result is on k
    assert why(rotary([q, k], [q, part(3, 2)])) == "shared"            # k's is on q
    assert why(rotary([k, part(6, 2)], [part(6, 2), k])) == "shared"   # swapped


def test_heads_first_and_tokens_first():
    """The same memory in both orders of axes, whole and in its two halves."""
    B, L, H, d = 1, 64, 8, 64
    q = view(B=B, L=L, H=H, d=d, stride_b=0)
    o = view(B=B, L=L, H=H, d=d, stride_b=0, stride_l=d, stride_h=L * d)
    assert why(attend(q, o)) == "shared"
    o.data += L * H * d * 2
    assert why(attend(q, o)) == "taken"
    # d = 128 in two halves, one of them tokens first
    a, b = view(B=1, L=9, H=3, d=64, stride_l=128 * 3, stride_h=128), view(B=1, L=9, H=3, d=64, data=PTR + 128, stride_l=128, stride_h=128 * 9)
    assert why(attend(a, b)) == "taken"
    b.data -= 16
    assert why(attend(a, b)) == "shared"


def units(v):
    """The 16-byte units of a bf16 view."""
    return {(v.data + 2 * (b * v.stride_b + l * v.stride_l + h * v.stride_h)) // 16 + u for b in range(v.B)
            for l in range(v.L) for h in range(v.H) for u in range(v.d // 8)}


@pytest.mark.parametrize("seed", range(8))
def test_against_the_sets_of_elements(seed):
    """Views with strides in any order, against the sets of their 16-byte units."""
    rng, seen = random.Random(seed), {"taken": 0, "shared": 0}
    for _ in range(300):
        shape = [rng.randint(1, 4) for _ in range(3)]
        d = 32

        def some():
            order, s, at = rng.sample(range(3), 3), [0, 0, 0], d + 8 * rng.randint(0, 9)
            for i in order:  # no element twice: the view may be written
                s[i] = at
                at = at * shape[i] + 8 * rng.randint(0, 9)
            return view(B=shape[0], L=shape[1], H=shape[2], d=d, data=PTR + 16 * rng.randint(0, 300), stride_b=s[0],
                        stride_l=s[1], stride_h=s[2])

        x, y = some(), some()
        if rng.random() < 0.3:  # read-only views may have one row for all
            x.stride_l = 0
        same = x.data == y.data and all(n == 1 or a == b for n, a, b in zip(
            shape, (x.stride_b, x.stride_l, x.stride_h), (y.stride_b, y.stride_l, y.stride_h)))
        want = "taken" if same or not units(x) & units(y) else "shared"
        assert why(attend(x, y)) == want
        assert why(rotary([x], [y])) == want
        seen[want] += 1
    assert min(seen.values()) > 20
