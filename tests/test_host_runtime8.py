"""The host side of 8-bit caches (argument checks, routes) on the stand-in for the CUDA runtime: no GPU, nothing runs."""
from test_host_runtime import host  # noqa: F401  (a fixture)

NEW8 = """
def new8(layers=1, hk=4, d=128, sink=4, vw=1000, tw=100, capacity=1500):
    h = vp()
    assert lib.svlm_cache_create8(C.byref(h), layers, hk, d, sink, vw, tw, capacity) == OK
    return h
"""


def test_alignment_of_device_pointers(host):  # noqa: F811
    """As for 16-bit caches, and beyond the shapes of their fast kernels too: the output is written by words there."""
    host(NEW8 + """
c = new8()
assert append(c, 40) == OK
ran()
for kw in (dict(K=P + 8), dict(V=P + 2)):
    assert append(c, 40, **kw) == ARG
for kw in (dict(Q=P + 2), dict(out=P + 8), dict(pos=P + 2)):
    assert attend(c, 40, **kw) == ARG and attend(c, 4, **kw) == ARG
for kw in (dict(Q=P + 1), dict(out=P + 2), dict(K=P + 3), dict(V=P + 1)):
    assert step(c, **kw) == ARG
wide, many = new8(hk=1, capacity=70000), new8(hk=1)     # more pages than the fast kernels' lists; more query heads a KV head than their rows
assert append(wide, 40) == OK and append(many, 40) == OK
ran()
for call in (lambda **kw: attend(wide, 1, hq=4, **kw), lambda **kw: attend(wide, 1, hq=9, **kw), lambda **kw: attend(wide, 5, hq=4, **kw), lambda **kw: attend(many, 1, hq=9, **kw)):
    for kw in (dict(out=P + 2), dict(out=P + 1), dict(Q=P + 1), dict(pos=P + 2)):
        assert call(**kw) == ARG, kw
    assert ran() == []
    assert call(Q=P + 2, out=P + 4) == OK
    assert any("rows8" in k for k in ran())
""")
