"""Caches that hold keys and values in 8 bits, where the kernels' paths meet: the statement, the comparison and its tolerances are
test_gpu_store8.py's."""
import numpy as np
import pytest
import torch

from harness import dev_to_f64
from paper_2510_09608_b200 import binding
from store8 import bf16
from test_gpu_store8 import Pair, close, to_dev

pytestmark = pytest.mark.gpu


def batched_step(ps, between=lambda out: None):
    """One generated token of every stream through all layers, in lock step; `between` gets each layer's output."""
    layers, hq, hk, d, n = ps[0].L, ps[0].hq, ps[0].hk, ps[0].d, len(ps)
    pos = np.stack([p.place([0]) for p in ps]).reshape(n)
    K, V = [p.normal(layers, 1, hk, d) for p in ps], [p.normal(layers, 1, hk, d) for p in ps]
    Q = bf16(ps[0].rng.standard_normal((layers, n, hq, d)))
    ty, qp = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.from_numpy(pos).cuda()
    k, v, q = ([to_dev(np.stack([x[l, 0] for x in xs])) for l in range(layers)] for xs in (K, V, [Q[:, None, i] for i in range(n)]))
    outs = []
    for l in range(layers):
        outs.append(binding.decode_step_batched([p.cache for p in ps], l, k[l], v[l], ty if l == 0 else None, qp, q[l]))
        between(outs[-1])
    for i, p in enumerate(ps):
        p.ref.append([0], pos[i:i + 1], K[i], V[i])
        for l in range(layers):
            close(dev_to_f64(outs[l])[i:i + 1], p.ref.attend(l, Q[l, i:i + 1], pos[i:i + 1]))
        assert p.cache.status() == binding.OK


@pytest.mark.parametrize("hq,hk,d", [(28, 4, 128), (4, 1, 64), (16, 2, 64)])
@pytest.mark.parametrize("text", [40, 56, 120])
def test_batched_steps_that_join_a_block_with_a_shift_of_its_own(hq, hk, d, text):
    """An answer goes on in the last block of an earlier one, whose tokens all stand off by what has left behind them; that block is the middle
    of a thread block's units (two of 16 tokens) and the one before it stands off as far.  Beside it a stream whose tokens are all off
    differently and one that has lost nothing, in the same launches."""
    ps = [Pair(500 + i, layers=3, hq=hq, hk=hk, d=d, sink=0, vw=16, tw=300) for i in range(3)]
    for rnd in range(2):
        ps[0].append([0] * text if rnd == 0 else [0] * 32)
        ps[0].append([1] * 64)
        ps[1].append([0, 1] * 28)
        ps[2].append([0] * 20 + [1] * 10)
        binding.evict_batched([ps[0].cache, ps[1].cache, ps[2].cache])
        for p in ps:
            p.ref.evict()
        for _ in range(4):
            batched_step(ps)
        for p in ps:
            p.check()


@pytest.mark.parametrize("text", [40, 56])
def test_all_layers_steps_that_join_a_block_with_a_shift_of_its_own(text):
    """The same in one launch for all layers of one stream."""
    p = Pair(520 + text, layers=3, hq=8, hk=2, d=128, sink=0, vw=16, tw=300)
    p.append([0] * text)
    p.append([1] * 64)
    p.evict()
    for _ in range(3):
        pos = p.place([0])
        K, V, Q = p.normal(3, 1, 2, 128), p.normal(3, 1, 2, 128), bf16(p.rng.standard_normal((3, 1, 8, 128)))
        zero = torch.zeros(1, dtype=torch.uint8, device="cuda")
        out = dev_to_f64(p.cache.decode_step(-1, to_dev(K), to_dev(V), zero, torch.from_numpy(pos).cuda(), to_dev(Q)))
        p.ref.append([0], pos, K, V)
        for l in range(3):
            close(out[l], p.ref.attend(l, Q[l], pos))
    p.check()


def tiny(p, n, hk, d, up):
    return bf16(p.normal(1, n, hk, d) * 2.0 ** up)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 5, 21, 40, 200])
def test_a_query_of_zeros_gives_the_mean(d, n):
    """One head's query is zero, another's next to nothing: equal weights for all stored tokens, whatever units the keys are in (blocks that
    are partly filled or missing in a pair; zero keys and tiny ones); the heads beside them are as they were."""
    for up in (0, -40, -110, None):
        p = Pair(600 + n, hq=8, hk=2, d=d, sink=2, vw=150, tw=100, capacity=512)
        K = None if up == 0 else np.zeros((1, n, 2, d)) if up is None else tiny(p, n, 2, d, up)
        p.append(p.rng.integers(0, 2, n), K=K)
        for n_q in (1, min(n, 3)):
            Q, pos = bf16(p.rng.standard_normal((n_q, 8, d))), p.pos[-n_q:]
            Q[:, 1], Q[:, 6] = 0, bf16(Q[:, 6] * 2.0 ** -122)
            got = dev_to_f64(p.cache.attend(0, to_dev(Q), torch.from_numpy(np.ascontiguousarray(pos)).cuda()))
            close(got, p.ref.attend(0, Q, pos))
        p.evict()
        pos, V = p.place([0]), p.normal(1, 1, 2, d)
        K = p.normal(1, 1, 2, d) if up == 0 else np.zeros((1, 1, 2, d)) if up is None else tiny(p, 1, 2, d, up)
        Q = np.zeros((1, 8, d))
        Q[0, 3] = bf16(p.rng.standard_normal(d))
        out = p.cache.decode_step(0, to_dev(K[0]), to_dev(V[0]), torch.zeros(1, dtype=torch.uint8, device="cuda"), torch.from_numpy(pos).cuda(), to_dev(Q))
        p.ref.append([0], pos, K, V)
        close(dev_to_f64(out), p.ref.attend(0, Q, pos))


@pytest.mark.parametrize("hq,hk,d,n", [(8, 2, 128, 150), (28, 4, 128, 140), (8, 2, 64, 200), (8, 1, 64, 300)])
def test_query_rows_of_zeros_in_a_long_chunk(hq, hk, d, n):
    """A chunk that goes over a widened layer, some of whose rows are zero (padding) or next to nothing: the mean of what they see, and the other
    rows as ever; over ordinary keys, tiny ones and zeros."""
    for up in (0, -60, None):
        p = Pair(660 + n, hq=hq, hk=hk, d=d, sink=2, vw=300, tw=200, capacity=900)
        p.append(p.rng.integers(0, 2, 170))
        p.evict()
        K = None if up == 0 else np.zeros((1, n, hk, d)) if up is None else tiny(p, n, hk, d, up)
        p.append(p.rng.integers(0, 2, n), K=K)
        Q, pos = bf16(p.rng.standard_normal((n, hq, d))), p.pos
        Q[3:20], Q[40, 1], Q[n - 1, hq - 1], Q[70] = 0, 0, 0, bf16(Q[70] * 2.0 ** -123)
        got = dev_to_f64(p.cache.attend(0, to_dev(Q), torch.from_numpy(np.ascontiguousarray(pos)).cuda()))
        assert p.cache.status() == binding.OK
        close(got, p.ref.attend(0, Q, pos))


@pytest.mark.parametrize("n_q", [1, 3])
def test_large_queries_over_small_keys(n_q):
    """Queries of 2^126 over keys of 400 * 2^-100: the product in the query's unit alone is no float, the scores (+-400 * 2^26 / sqrt(128)) are, and
    one token has all the weight.  (That direction turns with the position by less than 0.02.)"""
    p = Pair(640 + n_q, hq=8, hk=2, d=128, sink=2, vw=150, tw=100, capacity=512)
    K = np.zeros((1, 90, 2, 128))
    K[..., 63] = -400 * 2.0 ** -100
    K[0, 7, :, 63] *= -1
    p.append(p.rng.integers(0, 2, 90), K=bf16(K))
    Q, pos = np.zeros((n_q, 8, 128)), p.pos[-n_q:]
    Q[..., 63] = 2.0 ** 126
    got = dev_to_f64(p.cache.attend(0, to_dev(Q), torch.from_numpy(np.ascontiguousarray(pos)).cuda()))
    want = p.ref.attend(0, Q, pos)
    close(got, want)
    assert np.abs(want - p.ref.V[(7, 0)][np.arange(8) // 4]).max() == 0


@pytest.mark.parametrize("up", [8, 12, 16, 20])
@pytest.mark.parametrize("n", [20, 300])
def test_large_scores_leave_the_size_of_the_output_alone(n, up):
    """All values are 1.75, and so is every output, whatever the weights: scores of about 2^up; one token, appended or not, and a few rows."""
    p = Pair(650 + up, hq=8, hk=2, d=64, sink=2, vw=400, tw=200, capacity=900)
    V = np.ones((1, n, 2, 64)) * 1.75
    p.append(p.rng.integers(0, 2, n), V=V, K=bf16(p.normal(1, n, 2, 64) * 2.0 ** (up - 3)))
    for n_q in (1, 4):
        Q, pos = bf16(p.rng.standard_normal((n_q, 8, 64))), p.pos[-n_q:]
        got = dev_to_f64(p.cache.attend(0, to_dev(Q), torch.from_numpy(np.ascontiguousarray(pos)).cuda()))
        close(got, np.full(got.shape, 1.75))
    pos, K, Q = p.place([0]), bf16(p.normal(1, 1, 2, 64) * 2.0 ** (up - 3)), bf16(p.rng.standard_normal((1, 8, 64)))
    V = np.ones((1, 1, 2, 64)) * 1.75
    out = p.cache.decode_step(0, to_dev(K[0]), to_dev(V[0]), torch.zeros(1, dtype=torch.uint8, device="cuda"), torch.from_numpy(pos).cuda(), to_dev(Q))
    close(dev_to_f64(out), np.full((1, 8, 64), 1.75))


@pytest.mark.parametrize("hq,hk", [(28, 4), (8, 2)])
def test_steps_behind_one_that_gave_up_on_late_blocks(hq, hk):
    """Steps that wait for nothing (no polls) beside another stream's matrix products, so that some of a launch's blocks begin when others
    have given up on them: what those leave behind is not the next step's."""
    p = Pair(700 + hq, hq=hq, hk=hk, d=128, sink=4, vw=3000, tw=400, capacity=4096)
    p.append(p.rng.integers(0, 2, 2900))
    work, side = torch.randn(4096, 4096, device="cuda", dtype=torch.bfloat16), torch.cuda.Stream()
    into = torch.empty_like(work)
    ty = torch.zeros(1, dtype=torch.uint8, device="cuda")

    def step():
        pos, K, V, Q = p.place([0]), p.normal(1, 1, hk, 128), p.normal(1, 1, hk, 128), bf16(p.rng.standard_normal((1, hq, 128)))
        args = to_dev(K[0]), to_dev(V[0]), ty, torch.from_numpy(pos).cuda(), to_dev(Q)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(6):
                torch.mm(work, work, out=into)
        out = p.cache.decode_step(0, *args)
        p.ref.append([0], pos, K, V)
        return out, Q, pos
    for _ in range(12):
        p.cache.debug_set_wait_limit(0)
        step()
        p.cache.debug_set_wait_limit(1 << 20)
        out, Q, pos = step()
        close(dev_to_f64(out), p.ref.attend(0, Q, pos))
    assert p.cache.status() == binding.ERR_TIMEOUT               # sticky


@pytest.mark.parametrize("hq,hk,d,mrope", [(28, 4, 128, True), (8, 2, 64, False)])
def test_short_chunks_layer_by_layer(hq, hk, d, mrope):
    """Each layer's append directly behind the attention of the layer before it, as a model runs: few rows over the bytes, then a longer chunk, evictions
    and generated tokens between them; one cache and two at a time, whose rows differ in number."""
    ps = [Pair(800 + i, layers=3, hq=hq, hk=hk, d=d, sink=3, vw=120, tw=90, capacity=700, mrope=mrope) for i in range(2)]
    for rnd, n in enumerate((9, 21, 200, 1, 33, 12)):
        two = rnd % 3 == 1 or n == 12
        new = []
        for p in ps:
            types = p.rng.integers(0, 2, n).astype(np.uint8)
            pos = p.place(types)
            K, V, Q = p.normal(3, n, hk, d), p.normal(3, n, hk, d), bf16(p.rng.standard_normal((3, n, hq, d)))
            dev = to_dev(K), to_dev(V), to_dev(Q), torch.from_numpy(types).cuda(), torch.from_numpy(pos).cuda()
            new.append((types, pos, K, V, Q, dev))
        rows = [n, max(1, n - 3)]
        outs = []
        for l in range(3):
            for p, (_, _, _, _, _, (k, v, q, ty, at)) in zip(ps, new):
                p.cache.append(l, k[l], v[l], ty if l == 0 else None, at if l == 0 else None)
                if not two:
                    outs.append(p.cache.attend(l, q[l], at))
            if two:
                q = torch.cat([x[5][2][l][n - r:] for x, r in zip(new, rows)])
                at = torch.cat([x[5][4][n - r:] for x, r in zip(new, rows)])
                outs.append(binding.attend_batched_varlen([p.cache for p in ps], l, q, at, rows))
        for p, (types, pos, K, V, Q, _) in zip(ps, new):
            p.ref.append(types, pos, K, V)
            assert p.cache.status() == binding.OK
        for l in range(3):
            for i, (p, (_, pos, _, _, Q, _)) in enumerate(zip(ps, new)):
                if two:
                    close(dev_to_f64(outs[l][sum(rows[:i]):sum(rows[:i + 1])]), p.ref.attend(l, Q[l][n - rows[i]:], pos[n - rows[i]:]))
                else:
                    close(dev_to_f64(outs[2 * l + i]), p.ref.attend(l, Q[l], pos))
        for p in ps:
            if rnd % 2:
                p.evict()
            p.check()
            if hq // hk <= 8:
                p.step()


@pytest.mark.parametrize("d", [64, 128])
def test_two_chains_on_two_streams(d):
    """Generated tokens of two caches through all their layers, on a CUDA stream each and without a synchronisation between them: the blocks in which a
    launch's parts meet wait for others of theirs while another chain's launches take places on the GPU."""
    ps = [Pair(900 + i, layers=6, hq=8, hk=2, d=d, sink=4, vw=1500, tw=300, capacity=2200) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in ps]
    for p in ps:
        p.append(p.rng.integers(0, 2, 1600))
        p.evict()
    torch.cuda.synchronize()
    ty = torch.zeros(1, dtype=torch.uint8, device="cuda")
    steps = []
    for _ in range(8):
        for p in ps:
            pos = p.place([0])
            K, V, Q = p.normal(6, 1, 2, d), p.normal(6, 1, 2, d), bf16(p.rng.standard_normal((6, 1, 8, d)))
            steps.append((p, pos, K, V, Q, to_dev(K), to_dev(V), to_dev(Q), torch.from_numpy(pos).cuda(), torch.empty(6, 1, 8, d, dtype=torch.bfloat16, device="cuda")))
    torch.cuda.synchronize()
    for p, s in zip(ps, streams):
        p.cache.set_stream(s)
    for l in range(0, len(steps), 2):                        # a launch of the one, a launch of the other
        for layer in range(6):
            for p, _, _, _, _, k, v, q, at, out in steps[l:l + 2]:
                p.cache.decode_step(layer, k[layer], v[layer], ty if layer == 0 else None, at, q[layer], out[layer])
    torch.cuda.synchronize()
    for p, pos, K, V, Q, *_, out in steps:
        p.ref.append([0], pos, K, V)
        for layer in range(6):
            close(dev_to_f64(out[layer]), p.ref.attend(layer, Q[layer], pos))
    for p in ps:
        assert p.cache.status() == binding.OK
        p.cache.set_stream(torch.cuda.current_stream())
        p.check()


def test_batched_steps_with_projections_between_the_layers():
    """The layers' launches of a batched step begin early, but not as a chain: 4-bit projections of each layer's output run between them, as in a
    decoder.  (What is projected goes nowhere: the next layer's inputs are of the size that the tolerances are derived for.)"""
    import test_gpu_w4 as w4
    ps = [Pair(920 + i, layers=3, hq=8, hk=2, d=128, sink=4, vw=200, tw=100, capacity=700) for i in range(3)]
    for i, p in enumerate(ps):
        p.append(p.rng.integers(0, 2, 150 + 70 * i))
        p.evict()
    _, w, s = w4.inputs(3, 1024, 1536, 128, 5)
    for _ in range(4):
        batched_step(ps, between=lambda out: ps[0].cache.proj_w4(out.view(3, 1024), w, s))
    for p in ps:
        p.check()


@pytest.mark.parametrize("n_q", [[3, 3, 3], [9, 9, 9], [2, 40, 7]])
def test_batched_short_chunks_over_full_caches(n_q):
    """Questions of three streams over thousands of keys, of one length and of several: over the bytes and, by the number of rows and caches, over
    widened layers."""
    ps = [Pair(940 + i, hq=28, hk=4, d=128, sink=64, vw=3000, tw=300, capacity=3700, mrope=True, base=1e6) for i in range(3)]
    for p, n in zip(ps, n_q):
        p.append(np.r_[np.zeros(200), np.ones(2900)])
        p.append(np.r_[np.ones(300), np.zeros(60)])
        p.evict()
        p.append([0] * n)
    Q = [bf16(p.rng.standard_normal((n, 28, 128))) for p, n in zip(ps, n_q)]
    pos = torch.from_numpy(np.ascontiguousarray(np.concatenate([p.pos for p in ps]))).cuda()
    q, caches = to_dev(np.concatenate(Q)), [p.cache for p in ps]
    if len(set(n_q)) == 1:
        n = n_q[0]
        got = dev_to_f64(binding.attend_batched(caches, 0, q.view(3, n, 28, 128), pos.view(3, n, 3))).reshape(-1, 28, 128)
    else:
        got = dev_to_f64(binding.attend_batched_varlen(caches, 0, q, pos, n_q))
    at = 0
    for p, n, x in zip(ps, n_q, Q):
        assert p.cache.status() == binding.OK
        close(got[at:at + n], p.ref.attend(0, x, p.pos))
        at += n


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("up", [0, -70])
def test_a_giant_in_a_page_that_is_used_again(d, up):
    """The second layer's keys of new tokens arrive when the eviction is over; their page is one that a key of 1e30 (or ordinary ones, among keys that are far
    smaller since) has left.  What lies there of it is nobody's unit."""
    p = Pair(960, layers=2, hq=8, hk=2, d=d, sink=0, vw=200, tw=64, capacity=700)
    n = 130
    for rnd in range(5):
        types = np.ones(n, np.uint8)
        pos = p.place(types)
        K, V = bf16(p.normal(2, n, 2, d) * 2.0 ** (up if rnd else 0)), p.normal(2, n, 2, d)
        if rnd == 0:
            K[1, 5] = bf16(K[1, 5] * 1e30)
        p.cache.append(0, to_dev(K[0]), to_dev(V[0]), torch.from_numpy(types).cuda(), torch.from_numpy(pos).cuda())
        p.ref.append_meta(types, pos)
        p.ref.write(0, K[0], V[0])
        p.evict()
        p.cache.append(1, to_dev(K[1]), to_dev(V[1]))
        p.ref.write(1, K[1], V[1])
        if rnd < 2:                                          # (the giant is there)
            continue
        for n_q in (n, 3):
            Q = bf16(p.rng.standard_normal((n_q, 8, d)) * 2.0 ** -up)
            got = dev_to_f64(p.cache.attend(1, to_dev(Q), torch.from_numpy(np.ascontiguousarray(pos[-n_q:])).cuda()))
            close(got, p.ref.attend(1, Q, pos[-n_q:]))
    p.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("by", [1e8, 1e12, 1e30])
def test_a_giant_that_stays_when_another_has_left_its_block(d, by):
    """Two keys that are `by` times all others in one block, of which one is evicted: the other has all the weight of the queries it agrees with and none of
    the others', though its parts are far beyond f16 in the others' units.  (Its two directions turn with the position by 0.02 at most, and
    q.k is 0.8 or -0.8 of `by` before the rotation.)"""
    p = Pair(980, hq=8, hk=2, d=d, sink=0, vw=20, tw=400, capacity=768)
    K = p.normal(1, 190, 2, d)
    K[0, 3], K[0, 12] = bf16(K[0, 3] * by), 0
    K[0, 12, :, d // 2 - 1], K[0, 12, :, d // 2 - 2] = bf16(by), bf16(-0.1 * by)
    p.append([1] * 30 + [0] * 160, K=K)
    p.evict()
    p.check()
    for n_q in (1, 5, 140):
        Q, pos = bf16(p.rng.standard_normal((n_q, 8, d))), p.pos[-n_q:]
        sign = np.where(p.rng.integers(0, 2, (n_q, 8)), 1.0, -1.0)
        Q[..., d // 2 - 1], Q[..., d // 2 - 2] = sign, 2 * sign
        got = dev_to_f64(p.cache.attend(0, to_dev(Q), torch.from_numpy(np.ascontiguousarray(pos)).cuda()))
        close(got, p.ref.attend(0, Q, pos))


@pytest.mark.parametrize("bad", [np.nan, -np.inf])
@pytest.mark.parametrize("hq,hk,d,before,n", [(8, 2, 128, 150, 170), (8, 2, 64, 1500, 200), (28, 4, 128, 1700, 140)])
def test_a_value_that_is_not_finite_stays_out_of_the_rows_before_it_in_a_long_chunk(hq, hk, d, before, n, bad):
    """Values of a chunk that goes over a widened layer which are not finite, in several of its pages and in an earlier token: the rows that see them have
    NaN in those dims only, the rows of tokens before them are as ever.  One cache and two at once; the next layer and the next chunk have none of it."""
    G = hq // hk
    ps = [Pair(1000 + i, layers=2, hq=hq, hk=hk, d=d, sink=4, vw=before + 100, tw=100, capacity=before + 2 * n + 300) for i in range(2)]
    spots = [((3, 0, 7), (n // 2, 0, 7), (n // 2, 0, d // 2), (n // 2 + 1, hk - 1, d - 1), (n - 1, 0, 0)), ((0, 0, 1), (n - 2, hk - 1, 3))]
    news, Qs = [], []
    for p, where in zip(ps, spots):
        p.append(p.rng.integers(0, 2, before))
        p.evict()
        V = p.normal(2, n, hk, d)
        clean = V.copy()
        for tok, head, dim in where:
            V[0, tok, head, dim], clean[0, tok, head, dim] = bad, 0
        types = np.ones(n, np.uint8)
        types[-20:] = 0
        p.ref.append(types, pos := p.place(types), K := p.normal(2, n, hk, d), clean)
        p.pos = pos
        p.cache.append(-1, to_dev(K), to_dev(V), torch.from_numpy(types).cuda(), torch.from_numpy(pos).cuda())
        Qs.append(bf16(p.rng.standard_normal((2, n, hq, d))))
        lost = np.zeros((n, hq, d), bool)
        for tok, head, dim in where:
            lost[tok:, head * G:(head + 1) * G, dim] = True
        news.append((pos, lost))

    def see(got, i, layer):
        want, lost = ps[i].ref.attend(layer, Qs[i][layer], news[i][0]), news[i][1] if layer == 0 else np.zeros_like(news[i][1])
        assert ps[i].cache.status() == binding.OK and np.array_equal(np.isnan(got), lost)
        close(got[~lost], want[~lost])
    for layer in (0, 1, 0):
        for i, p in enumerate(ps):
            see(dev_to_f64(p.cache.attend(layer, to_dev(Qs[i][layer]), torch.from_numpy(news[i][0]).cuda())), i, layer)
        both = binding.attend_batched_varlen([p.cache for p in ps], layer, to_dev(np.concatenate([q[layer] for q in Qs])),
                                             torch.from_numpy(np.concatenate([x[0] for x in news])).cuda(), [n, n])
        for i in range(2):
            see(dev_to_f64(both[i * n:(i + 1) * n]), i, layer)
    for p in ps:                                             # the chunk's tokens are earlier ones now, and then gone
        for _ in range(3):
            p.append([1] * (before + 100) if before < 1000 else [1] * n)
            p.evict()
    if before < 1000:
        for p in ps:
            p.append([0] * 110 + [1] * n)
            p.evict()
            p.append([1] * n)
            p.attend(n)
