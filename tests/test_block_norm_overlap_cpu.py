"""Which outputs of the block norms may share memory with what: row outputs
with a row tensor, a parameter's gradient with the parameter, nothing else.
Against a runtime of imaginary devices: what is accepted launches nothing."""
from tests.fake_runtime import fake_library, run  # noqa: F401

FORWARD = """
T, D, ES = 64, 256, 2
SIZE = T * D * ES


def forward(gate_mode=3, ld=D, **at):
    # y, r, u, n, full gate and vectors a megabyte apart
    m = {k: (i + 1) << 20 for i, k in enumerate(
        ("y", "r", "u", "n", "gate", "w_post", "b_post", "w_pre", "b_pre"))}
    m.update(at)
    a = b.BlockNormArgs(m["y"], m["gate"] if gate_mode else None, m["w_post"], m["b_post"],
                        m["w_pre"], m["b_pre"], ld, ld, T, D, b.BF16, 1, 1, 1, gate_mode, 1.0, 1.0,
                        1e-5)
    return lib.ultramem_block_norm(C.byref(a), m["r"], m["u"], m["n"], None)


M = 1 << 20
assert forward() == b.OK
# in place
for at in (dict(u=2 * M, n=1 * M), dict(u=1 * M, n=2 * M), dict(u=5 * M), dict(n=5 * M),
           dict(u=2 * M)):
    assert forward(**at) == b.OK, at
launched = len(log())
# the outputs on one another
for at in (dict(u=4 * M), dict(u=4 * M + 2 * D * ES), dict(n=3 * M + SIZE - ES),
           dict(u=2 * M, n=2 * M)):
    assert forward(**at) == b.EINVAL, at
# an output that begins or ends inside an input, or on strided rows of one
for name, base in (("u", 1 * M), ("n", 2 * M), ("u", 5 * M)):
    for shift in (D * ES, -D * ES, SIZE - ES, ES - SIZE):
        assert forward(**{name: base + shift}) == b.EINVAL, (name, base, shift)
assert forward(ld=2 * D, u=2 * M) == b.EINVAL
assert forward(ld=2 * D, u=2 * M + D * ES) == b.EINVAL
# on parameters and on gates that are not row tensors
for vector in (6, 7, 8, 9):
    assert forward(u=vector * M) == b.EINVAL and forward(n=vector * M - D) == b.EINVAL
for mode in (1, 2):
    assert forward(gate_mode=mode, u=5 * M) == b.EINVAL
assert len(log()) == launched
# between the rows of a strided input there is room
assert forward(ld=T * D + D, u=1 * M + D * ES, r=1 << 30, n=1 << 31) == b.OK
assert forward(ld=T * D, u=1 * M + D * ES, r=1 << 30, n=1 << 31) == b.EINVAL
print("done")
"""

BACKWARD = """
T, D, ES = 64, 256, 2
SIZE = T * D * ES
M = 1 << 20
NAMES = ("y", "u", "du", "dn", "gate", "w_post", "b_post", "w_pre", "b_pre", "dy", "dr", "dgate",
         "dw_post", "db_post", "dw_pre", "db_pre", "ws")
AT = {k: (i + 1) * M for i, k in enumerate(NAMES)}
AT["ws"] = 1 << 30


def backward(gate_mode=3, ld=D, **at):
    m = dict(AT, **at)
    a = b.BlockNormArgs(m["y"], m["gate"], m["w_post"], m["b_post"], m["w_pre"], m["b_pre"], ld, ld,
                        T, D, b.BF16, 1, 1, 1, gate_mode, 1.0, 1.0, 1e-5)
    need = lib.ultramem_block_norm_backward_workspace(T, D)
    return lib.ultramem_block_norm_backward(
        C.byref(a), m["u"], m["du"], ld, m["dn"], ld, m["dy"], m["dr"], m["dgate"], m["dw_post"],
        m["db_post"], m["dw_pre"], m["db_pre"], m["ws"], need, None)


ROWS, OUT = ("y", "u", "du", "dn", "gate"), ("dy", "dr", "dgate")
assert backward() == b.OK
for o in OUT:
    for i in ROWS:
        assert backward(**{o: AT[i]}) == b.OK, (o, i)
VECTORS = {"dw_post": "w_post", "db_post": "b_post", "dw_pre": "w_pre", "db_pre": "b_pre"}
for o, i in VECTORS.items():
    assert backward(**{o: AT[i]}) == b.OK, o
for mode in (1, 2):
    assert backward(gate_mode=mode, dgate=AT["gate"]) == b.OK
launched = len(log())
for o in OUT:
    for i in ROWS:
        for shift in (D * ES, -D * ES):
            assert backward(**{o: AT[i] + shift}) == b.EINVAL, (o, i)
    for i in list(VECTORS.values()) + ["ws"]:
        assert backward(**{o: AT[i]}) == b.EINVAL, (o, i)
    for i in OUT:
        assert i == o or backward(**{o: AT[i] + 64}) == b.EINVAL, (o, i)
    assert backward(ld=2 * D, **{o: AT["y"]}) == b.EINVAL
for o, own in VECTORS.items():
    for i in NAMES:
        if i not in (o, own):
            assert backward(**{o: AT[i]}) == b.EINVAL, (o, i)
    assert backward(**{o: AT[own] + 4}) == b.EINVAL
for mode in (1, 2):
    for i in NAMES:
        if i not in ("dgate", "gate"):
            assert backward(gate_mode=mode, dgate=AT[i]) == b.EINVAL, (mode, i)
    assert backward(gate_mode=mode, dgate=AT["gate"] + 4) == b.EINVAL
assert len(log()) == launched
print("done")
"""


def test_forward(fake_library):  # noqa: F811
    run(fake_library, FORWARD)


def test_backward(fake_library):  # noqa: F811
    run(fake_library, BACKWARD)
