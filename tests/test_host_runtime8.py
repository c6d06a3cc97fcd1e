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


def test_positions_are_words(host):  # noqa: F811
    """Positions that do not begin at a word, of an append, of a projection that appends and of the general attention kernel: refused before anything runs."""
    host(NEW8 + """
for c in (new(), new8()):
    for layer in (-1, 0):
        for off in (1, 2, 3):
            assert lib.svlm_cache_append(c, layer, vp(P), vp(P), vp(P), vp(P + off), 40) == ARG
    assert ran() == [] and attend(c, 1) == ORDER                     # nothing was appended
    assert lib.svlm_cache_append(c, 0, vp(P), vp(P), vp(P + 1), vp(P + 4), 40) == OK
    ran()
c = new()
assert lib.svlm_qkv_append(c, 0, vp(P), vp(P), 128, 28, vp(P), vp(P + 2), 40, vp(P)) == ARG and ran() == []
wide = new(hk=1, capacity=70000)
assert append(wide, 40) == OK
ran()
for n, hq in ((40, 4), (1, 9)):
    for kw in (dict(pos=P + 2), dict(Q=P + 1), dict(out=P + 1)):
        assert attend(wide, n, hq=hq, **kw) == ARG
assert ran() == []
""")


def test_device_memory_is_what_the_header_lists(host):  # noqa: F811
    """28 layers of 4 heads of 128 fit into the parts that include/svlm.h names and 128 bytes a token for the metadata; no scratch of kernels that an
    8-bit cache never takes (9 MB here)."""
    host(NEW8 + """
L, H, D, capacity, sink = 28, 4, 128, 9800, 512
slots = 128 * ((sink + 127) // 128 + (capacity + 127) // 128 + 4)
bytes8 = 2 * L * H * slots * D + 4 * L * H * slots // 16
widened, turns, table = 2 * H * slots * D * 2, 2 * D * slots, 12 * 1024 * D // 2
fake.fake_alloc_limit(bytes8 + widened + turns + table + (3 << 20) + 128 * slots)
c = new8(L, H, D, sink, 8192, 512, capacity)
assert append(c, 40, layer=-1) == OK and step(c) == OK and attend(c, 1) == OK and attend(c, 1, hq=36) == OK and attend(c, 41) == OK
assert not any("decode" in k for k in ran())
""")


def test_a_captured_attention_is_reckoned_with_full_windows(host):  # noqa: F811
    """The attention call alone in a graph, captured on a nearly empty cache: its kernels are those of full windows already in that call."""
    host(NEW8 + """
c = new8(vw=8192, tw=512, capacity=9800)
assert append(c, 200) == OK
ran()
assert attend(c, 40) == OK
assert any("rows8" in k for k in ran())
fake.fake_capturing(1)
assert attend(c, 40) == OK
got = ran()
assert any("widen8" in k for k in got) and not any("rows8" in k for k in got), got
""")


def test_few_rows_or_a_widened_layer(host):  # noqa: F811
    """Which way a chunk goes over one cache and over several, of one length and of several; both sides were measured at each of these (us, bytes and widened)."""
    host(NEW8 + """
def fill(n, hk, d, keys, hq):
    cs = [new8(2, hk, d, 4, keys - 68, 64, keys + 600) for _ in range(n)]
    for c in cs:
        for at in range(0, keys, 512):
            assert append(c, min(512, keys - at), layer=-1) == OK
    return cs

def way(call):
    ran()
    assert call() == OK
    got = ran()
    few = any("rows8" in k for k in got)
    assert few != any("widen8" in k for k in got), got
    return few

for streams, hq, hk, d, keys, n, few in (
        (1, 28, 4, 128, 9216, 9, True), (1, 28, 4, 128, 9216, 73, False),           # 27 and 42, 141 and 43
        (4, 28, 4, 128, 9216, 4, True), (4, 28, 4, 128, 9216, 18, False),           # 45 and 73, 141 and 73
        (16, 28, 4, 128, 9216, 4, True), (16, 28, 4, 128, 9216, 9, False),          # 142 and 201, 276 and 201
        (16, 28, 4, 128, 336, 4, True), (16, 28, 4, 128, 336, 36, False),           # 15 and 28, 105 and 30
        (4, 16, 8, 64, 3100, 16, True), (4, 16, 8, 64, 3100, 64, False),            # 26 and 38, 87 and 38
        (1, 32, 8, 128, 9216, 16, True), (1, 32, 8, 128, 9216, 32, False),          # 45 and 48, 78 and 48
        (16, 4, 1, 64, 9216, 8, True), (16, 4, 1, 64, 9216, 32, False)):            # 35 and 49, 110 and 49
    cs = fill(streams, hk, d, keys, hq)
    one = lambda: attend(cs[0], n, hq=hq) if streams == 1 else lib.svlm_attend_batched(arr(cs), streams, 1, vp(P), vp(P), n, hq, vp(P))
    assert way(one) == few, (streams, hq, hk, d, keys, n)
    each = (C.c_int32 * streams)(*[n] * streams)
    assert way(lambda: lib.svlm_attend_batched_varlen(arr(cs), streams, 1, vp(P), vp(P), each, hq, vp(P))) == few
    for c in cs:
        lib.svlm_cache_destroy(c)

# sixteen caches one of which has a question of nine tokens, the others one token each; 28 layers in one call
cs = fill(16, 4, 128, 9216, 28)
each = (C.c_int32 * 16)(9, *[1] * 15)
assert way(lambda: lib.svlm_attend_batched_varlen(arr(cs), 16, 1, vp(P), vp(P), each, 28, vp(P)))
assert way(lambda: attend(cs[0], 9, layer=-1)) and not way(lambda: attend(cs[0], 73, layer=-1))
# an array with a hole in it is refused, not read
assert lib.svlm_attend_batched((vp * 2)(cs[0], None), 2, 0, vp(P), vp(P), 4, 28, vp(P)) == ARG
""")
