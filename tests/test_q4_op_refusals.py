"""What the operators that decode from a 4-bit cache refuse, and the host's account of pages: nothing is launched, so the
pointers are never followed and no GPU is needed."""
import ctypes as C
import random

import pytest

from test_context_op_refusals import b, _at, INVALID, SHAPE, WORKSPACE, UNSUPPORTED, TOO_LARGE  # noqa: F401

ROPE = dict(layout=0, rot_dim=64, scaling=0, base=1e4, factor=2.0, orig_ctx=4096.0, low=1.0, high=32.0, magnitude=0.0)
TURN = dict(dtype=1, q=_at(0), q_ld=512, k=_at(1), k_ld=256, pos=_at(4), n=3, nq=4, nkv=2, hd=128, rope=None, q_out=_at(5),
            q_out_ld=512, k_out=_at(6), k_out_ld=256, stream=None)
PAGE = 64 * 72 * 2 * 2                      # 2 kv heads of 128
APPEND = dict(dtype=1, k=_at(0), k_ld=256, v=_at(1), v_ld=256, R=3, off=None, lens=_at(2), S=3, table=_at(3), table_ld=4, width=4, nkv=2,
              hd=128, pool=_at(5), page_ld=PAGE, n_pages=20, stream=None)
READ = dict(dtype=1, pool=_at(5), page_ld=PAGE, n_pages=20, table=_at(3), table_ld=4, width=4, off=None, lens=_at(2), S=3, R=3, nkv=2,
            hd=128, k_out=_at(0), v_out=_at(1), stream=None)
COPY = dict(pool=_at(0), layer_ld=20 * PAGE, page_ld=PAGE, page_bytes=PAGE, L=2, n_pages=20, src=_at(5), dst=_at(6), n=3, stream=None)
ATTEND = dict(dtype=1, q=_at(0), q_ld=512, R=3, pool=_at(1), page_ld=PAGE, n_pages=20, table=_at(2), table_ld=4, width=4, lens=_at(3),
              off=None, S=3, nq=4, nkv=2, hd=128, out=_at(4), lse=_at(5), scratch=_at(6), scratch_bytes=1 << 23, stream=None)
LINEAR = dict(dtype=1, x=_at(0), x_ld=256, w=_at(1), w_bytes=16 * 4 * 576, y=_at(3), M=3, N=256, K=256, scratch=None,
              scratch_bytes=0, stream=None)
RESIDUAL = dict(dtype=1, x=_at(0), x_ld=256, w=_at(1), w_bytes=16 * 4 * 576, h=_at(3), out=_at(4), M=3, N=256, K=256,
                scratch=None, scratch_bytes=0, stream=None)
PACK = dict(codes=_at(0), meta=_at(1), N=256, K=256, packed=_at(2), stream=None)


@pytest.mark.parametrize("change,rope,code", [
    (dict(dtype=3), {}, UNSUPPORTED), (dict(hd=100), {}, UNSUPPORTED), (dict(hd=264), {}, UNSUPPORTED), (dict(n=-1), {}, INVALID),
    (dict(nkv=-1), {}, INVALID), (dict(q=None), {}, INVALID), (dict(pos=None), {}, INVALID), (dict(k_out=None), {}, INVALID),
    (dict(q_ld=504), {}, SHAPE), (dict(q=_at(0) + 2), {}, INVALID), (dict(k_ld=257), {}, INVALID), (dict(k_out=_at(5) + 256), {}, INVALID),
    (dict(q_out=_at(0), q_out_ld=768), {}, INVALID), (dict(q_out=_at(1)), {}, INVALID), (dict(k_out=_at(4)), {}, INVALID),
    ({}, dict(layout=2), UNSUPPORTED), ({}, dict(scaling=5), UNSUPPORTED), ({}, dict(scaling=-1), UNSUPPORTED), ({}, dict(rot_dim=0), SHAPE),
    ({}, dict(rot_dim=63), SHAPE), ({}, dict(rot_dim=130), SHAPE), ({}, dict(rot_dim=2, scaling=2), SHAPE), ({}, dict(base=0.0), INVALID),
    ({}, dict(base=float("nan")), INVALID), ({}, dict(magnitude=-1.0), INVALID), ({}, dict(scaling=1, factor=0.0), INVALID),
    ({}, dict(scaling=3, orig_ctx=0.0), INVALID), ({}, dict(scaling=3, low=4.0, high=4.0), INVALID), ({}, dict(scaling=4, low=0.0), INVALID),
    ({}, dict(scaling=4, base=1.0), INVALID), ({}, dict(scaling=4, factor=float("inf")), INVALID),
])
def test_rope_scaled_refuses(b, change, rope, code):  # noqa: F811
    d = b.RopeDesc(*{**ROPE, **rope}.values())
    assert b.lib.akvs_op_rope_scaled(*{**TURN, "rope": C.addressof(d), **change}.values()) == code


def test_rope_scaled_nothing_to_do(b):  # noqa: F811
    desc = b.RopeDesc(*ROPE.values())
    d = C.addressof(desc)
    assert b.lib.akvs_op_rope_scaled(*{**TURN, "rope": None}.values()) == INVALID
    assert b.lib.akvs_op_rope_scaled(*{**TURN, "rope": d, "n": 0, "q": None}.values()) == 0
    assert b.lib.akvs_op_rope_scaled(*{**TURN, "rope": d, "nq": 0, "nkv": 0}.values()) == 0
    with pytest.raises(b.AkvsError):
        b.Rope(1e4, 64, layout="third")


COMMON = [(dict(dtype=7), UNSUPPORTED), (dict(hd=96), UNSUPPORTED), (dict(R=-1), INVALID), (dict(S=-1), INVALID), (dict(width=-1), INVALID),
          (dict(n_pages=-1), INVALID), (dict(nkv=0), SHAPE), (dict(R=2), SHAPE), (dict(lens=None), INVALID), (dict(table=None), INVALID),
          (dict(pool=None), INVALID), (dict(table_ld=3), SHAPE), (dict(page_ld=PAGE - 16), SHAPE), (dict(page_ld=PAGE + 8), INVALID),
          (dict(pool=_at(5) + 8), INVALID)]


@pytest.mark.parametrize("change,code", COMMON + [
    (dict(k=None), INVALID), (dict(k_ld=128), SHAPE), (dict(v_ld=257), INVALID), (dict(v=_at(1) + 4), INVALID), (dict(k=_at(5)), INVALID),
    (dict(pool=_at(2)), INVALID), (dict(off=_at(5) + 64), INVALID)])
def test_append_refuses(b, change, code):  # noqa: F811
    assert b.lib.akvs_op_pages_append(*{**APPEND, **change}.values()) == code


@pytest.mark.parametrize("change,code", COMMON + [
    (dict(k_out=None), INVALID), (dict(v_out=_at(1) + 8), INVALID), (dict(v_out=_at(0) + 256), INVALID), (dict(k_out=_at(5)), INVALID),
    (dict(v_out=_at(3)), INVALID)])
def test_read_refuses(b, change, code):  # noqa: F811
    assert b.lib.akvs_op_pages_read(*{**READ, **change}.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(L=-1), INVALID), (dict(n=-1), INVALID), (dict(pool=None), INVALID), (dict(src=None), INVALID), (dict(page_ld=PAGE - 16), SHAPE),
    (dict(layer_ld=PAGE), SHAPE), (dict(page_bytes=40, page_ld=48), INVALID), (dict(pool=_at(0) + 8), INVALID), (dict(layer_ld=20 * PAGE + 8), INVALID),
    (dict(src=_at(0) + 32), INVALID), (dict(n=65536), TOO_LARGE)])
def test_copy_refuses(b, change, code):  # noqa: F811
    assert b.lib.akvs_op_pages_copy(*{**COPY, **change}.values()) == code


@pytest.mark.parametrize("change,code", [
    (c if "pool" not in c or c["pool"] is None else dict(pool=_at(1) + 8), e) for c, e in COMMON] + [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(lse=None), INVALID), (dict(q_ld=256), SHAPE), (dict(q_ld=516), INVALID),
    (dict(nq=5), SHAPE), (dict(nq=258), SHAPE), (dict(scratch=None), WORKSPACE), (dict(scratch=_at(6) + 16), WORKSPACE),
    (dict(scratch_bytes=64), WORKSPACE), (dict(out=_at(0)), INVALID), (dict(lse=_at(3)), INVALID), (dict(scratch=_at(1)), INVALID),
    (dict(out=_at(6)), INVALID), (dict(R=1 << 30), TOO_LARGE), (dict(width=1 << 26, table_ld=1 << 26), TOO_LARGE)])
def test_attention_refuses(b, change, code):  # noqa: F811
    assert b.lib.akvs_op_attention_pages(*{**ATTEND, **change}.values()) == code


@pytest.mark.parametrize("change,code", [
    (dict(dtype=5), UNSUPPORTED), (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(K=200), SHAPE), (dict(x=None), INVALID),
    (dict(w=None), INVALID), (dict(x_ld=248), SHAPE), (dict(x_ld=257), INVALID), (dict(w_bytes=16 * 4 * 576 - 1), SHAPE),
    (dict(x=_at(0) + 8), INVALID), (dict(w=_at(1) + 8), INVALID)])
def test_linear_refuses(b, change, code):  # noqa: F811
    assert b.lib.akvs_op_linear_q4(*{**LINEAR, **change}.values()) == code
    assert b.lib.akvs_op_linear_q4_residual(*{**RESIDUAL, **change}.values()) == code


def test_linear_refuses_outputs(b):  # noqa: F811
    f, r = b.lib.akvs_op_linear_q4, b.lib.akvs_op_linear_q4_residual
    for change in (dict(y=None), dict(y=_at(0)), dict(y=_at(1) + 64), dict(y=_at(3) + 1)):
        assert f(*{**LINEAR, **change}.values()) == INVALID
    for change in (dict(h=None), dict(out=None), dict(out=_at(0)), dict(out=_at(3) + 4), dict(h=_at(3) + 2), dict(out=_at(4) + 2)):
        assert r(*{**RESIDUAL, **change}.values()) == INVALID
    assert f(*{**LINEAR, "M": 0, "x": None}.values()) == 0
    for change, code in ((dict(N=0), INVALID), (dict(K=100), SHAPE), (dict(codes=None), INVALID), (dict(packed=_at(2) + 8), INVALID),
                         (dict(meta=_at(1) + 2), INVALID), (dict(packed=_at(0)), INVALID)):
        assert b.lib.akvs_op_linear_q4_pack(*{**PACK, **change}.values()) == code


def test_sizes(b):  # noqa: F811
    assert b.page_bytes(2, 128) == PAGE and b.page_bytes(1, 64) == 4608 and b.page_bytes(0, 64) == b.page_bytes(1, 96) == -1
    f = b.lib.akvs_linear_q4_bytes
    assert f(16, 64) == 1152 and f(17, 192) == 4 * 1152 and f(0, 64) == f(5, 65) == -1
    assert f(2 ** 31 - 256, 64) == 1152 * (2 ** 27 - 16) and f(2 ** 31 - 255, 64) == f(2 ** 31 - 1, 64) == -1
    f = b.lib.akvs_op_attention_pages_scratch_bytes
    assert f(3, 3, 5, 2, 128) == f(-1, 3, 4, 2, 128) == f(3, 3, 4, 2, 32) == -1
    last = 0
    for R, S in ((0, 0), (1, 1), (2, 1), (2, 2), (7, 2), (7, 7), (8, 7), (4000, 7), (4000, 4000)):
        n = f(R, S, 40, 8, 128)
        assert n >= last
        last = n


def test_linear_scratch(b):  # noqa: F811
    """It never shrinks when a call grows, in rows, columns or features; where there is one, it is asked for."""
    f = b.lib.akvs_op_linear_q4_scratch_bytes
    assert f(1, -1, 64, 64) == f(3, 1, 64, 64) == f(1, 1, 64, 63) == -1 and f(1, 0, 64, 64) == f(0, 500, 64, 64) == 0
    Ms, Ns, Ks = (1, 4, 8, 9, 16, 17, 32, 33, 64, 65, 200), (16, 4096, 28672, 60000), (64, 4096, 14336, 27648)
    size = {(M, N, K): f(2, M, N, K) for M in Ms for N in Ns for K in Ks}
    for (M, N, K), n in size.items():
        assert all(n <= n2 for (M2, N2, K2), n2 in size.items() if M2 >= M and N2 >= N and K2 >= K)
    big = dict(M=20, x=_at(0), w=_at(1), y=_at(3))
    need = f(1, 20, 256, 256)
    assert need > 0
    for change, code in ((dict(), WORKSPACE), (dict(scratch=_at(5), scratch_bytes=need - 1), WORKSPACE),
                         (dict(scratch=_at(5) + 16, scratch_bytes=need), WORKSPACE), (dict(scratch=_at(1), scratch_bytes=need), INVALID),
                         (dict(scratch=_at(3) - 256, scratch_bytes=need), INVALID)):
        assert b.lib.akvs_op_linear_q4(*{**LINEAR, **big, **change}.values()) == code


def test_host_tensors_are_refused(b):  # noqa: F811
    import torch
    x, i = torch.zeros((2, 2, 64)), torch.zeros(2, dtype=torch.int32)
    pool, table = torch.zeros((3, b.page_bytes(2, 64)), dtype=torch.uint8), torch.zeros((2, 1), dtype=torch.int32)
    for call in (lambda: b.op_rope_scaled(x, x, i, b.Rope(1e4, 64)), lambda: b.op_pages_append(x, x, pool, table, i),
                 lambda: b.op_pages_read(pool, table, i, x, x.clone()), lambda: b.op_pages_copy(pool[None], i, i),
                 lambda: b.op_attention_pages(x, pool, table, i, 2), lambda: b.LinearQ4(torch.zeros(4, 64))):
        with pytest.raises(b.AkvsError):
            call()


# --------------------------------------------------------------------------- the account of pages

@pytest.fixture
def pool(b, monkeypatch):  # noqa: F811
    """A pool whose pages hold one number in place of their tokens."""
    import paper_2607_21604_b200.pages as pages
    monkeypatch.setattr(pages.binding, "op_pages_copy", lambda p, s, d: p.__setitem__((slice(None), d.long()), p[:, s.long()]))
    return pages.PagePool(2, 12, 1, 64, device="cpu")


def _check(p):
    held = {}
    for s, ps in p.pages.items():
        assert len(ps) == -(-p.length[s] // 64)
        for x in ps:
            held[x] = held.get(x, 0) + 1
    assert [held.get(x, 0) for x in range(len(p.users))] == p.users
    assert sorted(p.free) == [x for x in range(len(p.users)) if not p.users[x]]


def test_pool_branches(pool):
    a = pool.open()
    pool.grow([a], 70)
    assert pool.pages[a] == [0, 1] and pool.length[a] == 70
    pool.pool[:, 1] = 7
    x, y = pool.fork(a, 2)
    _check(pool)
    pool.grow([a, x, y])                              # all three go on in the shared last page: two copies
    assert pool.pages[a][0] == pool.pages[x][0] == pool.pages[y][0] == 0
    assert len({pool.pages[s][1] for s in (a, x, y)}) == 3 and (pool.pool[:, [pool.pages[s][1] for s in (a, x, y)]] == 7).all()
    _check(pool)
    table, lens = pool.table([x, a])
    assert table.tolist() == [pool.pages[x], pool.pages[a]] and lens.tolist() == [71, 71]
    pool.cut(x, 64)
    assert pool.pages[x] == [0]
    pool.grow([x], 64)                                # a full last page is shared as it is
    assert pool.pages[x][0] == 0 and pool.length[x] == 128
    _check(pool)


def test_pool_runs_out(pool, b):  # noqa: F811
    a, c = pool.open(), pool.open()
    pool.grow([a, c], [64 * 6, 64 * 6])
    state = (dict(pool.pages), dict(pool.length), list(pool.users))
    with pytest.raises(b.AkvsError):
        pool.grow([a, c], [0, 1])
    assert state == (pool.pages, pool.length, pool.users)
    pool.grow([a], 0)
    pool.close(c)
    pool.grow([a], 1)
    _check(pool)
    for bad in (lambda: pool.cut(a, -1), lambda: pool.cut(a, 10 ** 4), lambda: pool.grow([a, a]), lambda: pool.grow([a], -1), lambda: pool.grow([a], [1, 2])):
        with pytest.raises(b.AkvsError):
            bad()


def test_pool_any_history(pool, b):  # noqa: F811
    """Random histories: what a page holds follows its sequence, through branches and moves."""
    rng = random.Random(5)
    want = {}                                         # sequence -> number of every page
    for step in range(600):
        seqs = list(want)
        act = rng.choice(("open", "grow", "grow", "fork", "close", "compact", "cut"))
        if act == "open" and len(seqs) < 6:
            want[pool.open()] = []
        elif act == "grow" and seqs:
            s, n = rng.choice(seqs), rng.randint(1, 130)
            try:
                pool.grow([s], n)
            except b.AkvsError:
                continue
            for i in range(len(want[s]), len(pool.pages[s])):
                want[s].append(step % 251)
                pool.pool[:, pool.pages[s][i]] = step % 251
        elif act == "fork" and seqs:
            s = rng.choice(seqs)
            for t in pool.fork(s, rng.randint(1, 2)):
                want[t] = list(want[s])
        elif act == "close" and seqs:
            s = rng.choice(seqs)
            pool.close(s)
            del want[s]
        elif act == "cut" and seqs:
            s = rng.choice(seqs)
            pool.cut(s, rng.randint(0, pool.length[s]))
            del want[s][len(pool.pages[s]):]
        elif act == "compact":
            pool.compact()
            assert all(not u for u in pool.users[sum(1 for u in pool.users if u):])
        _check(pool)
        for s, pages in want.items():
            assert pool.pool[0, pool.pages[s], 0].tolist() == pool.pool[1, pool.pages[s], 5].tolist() == pages


def _state(p):
    return {s: list(x) for s, x in p.pages.items()}, dict(p.length), list(p.users), list(p.free)


def test_pool_keeps_its_account_when_a_copy_is_refused(pool, b, monkeypatch):  # noqa: F811
    """A call whose copy is refused changes nothing and can be repeated."""
    import paper_2607_21604_b200.pages as pages
    a, gap = pool.open(), pool.open()
    pool.grow([a], 70)
    pool.grow([gap], 130)
    pool.pool[:, 1] = 7
    (x,) = pool.fork(a)
    state, copy = _state(pool), pages.binding.op_pages_copy

    def refuse(*_):
        raise b.AkvsError(-1, "akvs_op_pages_copy")
    monkeypatch.setattr(pages.binding, "op_pages_copy", refuse)
    with pytest.raises(b.AkvsError):
        pool.grow([a, x], [100, 1])
    assert _state(pool) == state
    monkeypatch.setattr(pages.binding, "op_pages_copy", copy)
    pool.grow([a, x], [100, 1])
    assert (pool.length[a], pool.length[x]) == (170, 71)
    assert pool.pages[a][1] != pool.pages[x][1] and (pool.pool[:, [pool.pages[s][1] for s in (a, x)]] == 7).all()
    _check(pool)
    pool.close(gap)                                   # pages 2 to 4: those behind them would move
    state = _state(pool)
    monkeypatch.setattr(pages.binding, "op_pages_copy", refuse)
    with pytest.raises(b.AkvsError):
        pool.compact()
    assert _state(pool) == state


def test_pool_fork_of_no_sequence(pool):
    """Nothing is opened for a sequence that there is not."""
    a = pool.open()
    pool.grow([a], 5)
    state = _state(pool)
    with pytest.raises(KeyError):
        pool.fork(a + 1, 2)
    assert _state(pool) == state


def test_linear_beyond_a_grid(b):  # noqa: F811
    """More blocks than a launch has: refused by both, the call and its scratch size.  Sizes that a GPU holds are not."""
    f = b.lib.akvs_op_linear_q4_scratch_bytes
    last = 2 ** 31 - 1
    for dt, M, N, K in ((0, last, 2 ** 30, 64), (1, last, 2 ** 30, 64), (2, 2 ** 30, 2 ** 31 - 256, 64), (1, last, 64, 2 ** 31 - 64)):
        assert f(dt, M, N, K) == -1
        change = dict(dtype=dt, M=M, N=N, K=K, x_ld=K, w_bytes=2 ** 62, x=_at(0), w=2 ** 62, y=2 ** 60, scratch=_at(1), scratch_bytes=2 ** 62)
        assert b.lib.akvs_op_linear_q4(*{**LINEAR, **change}.values()) == TOO_LARGE
    for dt, M, N, K in ((0, 9, 2 ** 31 - 256, 64), (0, 2 ** 24, 64, 64), (1, 17, 2 ** 31 - 256, 64), (2, 2 ** 26, 1, 64), (0, 8, 2 ** 31 - 256, 64)):
        assert f(dt, M, N, K) >= 0
