"""Which arguments of the paged calls may share memory: out with q, nothing
else that a call writes.  Against a runtime of imaginary devices: what is
accepted launches nothing."""
from tests.fake_runtime import fake_library, run  # noqa: F401

PLAN = """
M = 1 << 20
R, W, F, T = 300, 7, 900, 5000
NAMES = ("ctx", "new", "table", "pages", "count", "q_start", "kv", "slots", "left", "balance")
SIZE = dict(ctx=R, new=R, table=R * W, pages=F, count=1, q_start=R + 1, kv=R, slots=T, left=1,
            balance=1)
AT = {k: (i + 1) * M for i, k in enumerate(NAMES)}


def plan(**at):
    m = dict(AT, **at)
    return lib.ultramem_paged_plan(m["ctx"], m["new"], R, 16, m["table"], W, m["pages"], m["count"],
                                   F, T, m["q_start"], m["kv"], m["slots"], m["left"], m["balance"],
                                   None)


assert plan() == b.OK and plan(left=None) == b.OK
assert plan(count=AT["pages"] + 4 * F, left=AT["pages"] - 4) == b.OK      # neighbours
launched = len(log())
for o in ("table", "q_start", "kv", "slots", "left", "balance"):
    for i in NAMES:
        if i != o:
            for at in (AT[i], AT[i] + 4 * SIZE[i] - 4, AT[i] - 4 * SIZE[o] + 4):
                assert plan(**{o: at}) == b.EINVAL, (o, i)
assert len(log()) == launched
print("done")
"""

ATTENTION = """
M = 1 << 20
T, H, D, W = 24, 8, 64, 5
ROW = H * D * 2
NAMES = ("q", "q_start", "kv", "table", "out", "lse")
AT = {k: (i + 1) * M for i, k in enumerate(NAMES)}
AT["ws"] = 1 << 30
SIZE = dict(q=T * ROW, q_start=16, kv=12, table=12 * W, out=T * ROW, lse=4 * T * H)


def attention(stride=H * D, max_new=8, **at):
    m = dict(AT, **at)
    c = b.KVCache(1 << 35, 1 << 36, 64, 2, 16, D, b.BF16)
    need = lib.ultramem_paged_attention_workspace(b.BF16, H, 2, D, max_new)
    return lib.ultramem_paged_attention(C.byref(c), m["q"], stride, H, m["q_start"], m["kv"],
                                        m["table"], W, 3, T, max_new, 1.0, m["out"], m["lse"],
                                        m["ws"], need, None)


for max_new in (1, 8):
    assert attention(max_new=max_new) == b.OK and attention(max_new=max_new, lse=None) == b.OK
    assert attention(max_new=max_new, out=AT["q"]) == b.OK
assert attention(stride=(T + 1) * H * D, out=AT["q"] + ROW, lse=1 << 31) == b.OK   # between rows
launched = len(log())
assert attention(stride=2 * H * D, out=AT["q"]) == b.EINVAL
for o in ("out", "lse"):
    for i in NAMES:
        if i != o:
            for at in (AT[i], AT[i] + SIZE[i] - 4, AT[i] - SIZE[o] + 4):
                if (o, i, at) != ("out", "q", AT["q"]):
                    assert attention(**{o: at}) == b.EINVAL, (o, i)
for i in NAMES:
    assert attention(ws=AT[i]) == b.EINVAL and attention(ws=AT[i] - 4096) == b.EINVAL, i
assert len(log()) == launched
print("done")
"""


def test_plan(fake_library):  # noqa: F811
    run(fake_library, PLAN)


def test_attention(fake_library):  # noqa: F811
    run(fake_library, ATTENTION)
