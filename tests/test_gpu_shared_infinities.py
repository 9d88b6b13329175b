"""Infinities and NaN in V of what shared prompts and own lists hold, at lengths whose last 32 keys are not whole: outputs have them where they are,
and only there, whichever form a group's size, type or query grouping takes."""
import pytest
import torch


from test_gpu_shared import Shared

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def expect(s, mark):
    """mark(V, PV): puts values that are not finite where they are wanted; every other output is the one without them."""
    s.run()
    clean, lse, score = (t.clone() for t in (s.batch.out, s.batch.lse, s.batch.score))
    s.batch.score.copy_(torch.from_numpy(s.score0))
    want = {}
    for (b, head, e), x in mark(s).items():
        for j in range(head * s.G, (head + 1) * s.G):
            want[b, j, e] = x
    s.run()
    out = s.batch.out.clone()
    for at, x in want.items():
        assert (out[at].isnan() if x != x else out[at] == x), (at, float(out[at]), x)
        out[at] = clean[at]
    assert torch.equal(out, clean) and torch.equal(s.batch.lse, lse) and torch.equal(s.batch.score, score)


FORMS = [(2, 64, "bf16", 0), (2, 128, "bf16", 0), (2, 64, "f32", 0), (2, 128, "f32", 0), (2, 64, "bf16", 3), (2, 128, "bf16", 8)]


@pytest.mark.parametrize("h,D,dtype,G", FORMS)
@pytest.mark.parametrize("members", [[3, 2], [40, 5]])
@pytest.mark.parametrize("prompts", [[33, 1], [70, 127], [200, 32], [501, 90]])
def test_in_the_last_slots_of_a_prompt(h, D, dtype, G, members, prompts):
    s = Shared(members, prompts, [20 + b % 7 for b in range(sum(members))], h, D, dtype, G)

    def mark(s):
        want = {}
        for g, m in enumerate(prompts):
            for head in range(h):
                s.PV[g, head, m - 1, 3] = INF if head else -INF
                s.PV[g, head, m // 2, D - 1] = NAN
                for b in range(s.members[g], s.members[g + 1]):
                    want[b, head, 3], want[b, head, D - 1] = INF if head else -INF, NAN
        return want

    expect(s, mark)


@pytest.mark.parametrize("h,D,dtype,G", FORMS)
@pytest.mark.parametrize("lists", [[1, 2, 5, 33, 64], [31, 63, 95, 130, 300]])
@pytest.mark.parametrize("new_at", [-1, 0, 4])
@pytest.mark.parametrize("place", ["last", "first"])
def test_in_an_own_list(h, D, dtype, G, lists, new_at, place):
    """At the list's last key that is resident, or its first one: the rows that stand in for keys past the end and for the query token."""
    s = Shared([2, 3], [40, 7], lists, h, D, dtype, G, new_at=new_at)

    def mark(s):
        want = {}
        for b, sel in enumerate(s.sel):
            resident = sel[sel != s.pending[b]]
            if not len(resident):
                continue
            slot = resident[-1 if place == "last" else 0]
            for head in range(h):
                s.V[b, head, slot, 5], s.V[b, head, slot, 6] = (INF, -INF) if head else (-INF, INF)
                want[b, head, 5], want[b, head, 6] = (INF, -INF) if head else (-INF, INF)
        return want

    expect(s, mark)
