"""The extension's calls of the cache and of attention against their ctypes forms: the same arguments reach the library in every form of a call
that these take, and the same exceptions leave it."""
import ctypes

import pytest

import paper_2512_17970_amd as cg
from paper_2512_17970_amd import binding

vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
cp, ap, tp = ctypes.POINTER(cg.KvCache), ctypes.POINTER(cg.AppendDesc), ctypes.POINTER(cg.AttnDesc)
TAKES = {"kv_append": (cp, ap, vp, vp, vp, vp, vp, vp, vp, vp, vp), "kv_gather": (cp, i32, vp, vp, vp, vp), "attn_decode": (cp, tp, vp, vp, vp, sz),
         "attn_prompt": (tp, vp, vp, vp, vp, vp, vp, vp, sz)}
CACHE = cg.KvCache(kv_heads=3, head_dim=64, dtype=1, page_size=16, scale_block=4, num_pages=77, num_seqs=5, max_pages=9, k=0x1000, v=0x2000, page_table=0x50, kv_lens=0x60)
APPEND, ATTN = cg.AppendDesc(tokens=4, q_heads=6, rotary_dim=32), cg.AttnDesc.make(6, 3, 64, num_seqs=5, total_q=5, max_kv=99, scale=0.5)
GIVEN = {cp: CACHE, ap: APPEND, tp: ATTN}


class Tensor:
    def __init__(self, at):
        self.at = at

    def data_ptr(self):
        if isinstance(self.at, BaseException):
            raise self.at
        return self.at


@pytest.fixture()
def calls():
    """Both forms with the library's functions replaced by ones that note what they are given and return `status`."""
    lib, seen, status, kept = binding.load(), [], [0], []

    def noting(takes):
        def f(*args):
            seen.append([bytes(a[0]) if t in GIVEN else a for a, t in zip(args, (*takes, vp))])
            return status[0]
        return ctypes.CFUNCTYPE(ctypes.c_int, *takes, vp)(f)

    names = ["codegemm_" + n for n in TAKES]
    real = [getattr(lib, n) for n in names]
    address = lambda f: ctypes.cast(f, vp).value  # noqa: E731
    for n, takes in TAKES.items():
        kept.append(noting(takes))
        setattr(lib, "codegemm_" + n, kept[-1])
    binding._calls.use_attention(*map(address, kept))
    yield seen, status
    for n, f in zip(names, real):
        setattr(lib, n, f)
    binding._calls.use_attention(*map(address, real))


def outcome(f, seen, *args, **kwargs):
    del seen[:]
    try:
        got = f(*args, **kwargs)
    except BaseException as e:
        got = (type(e), str(e))
    return got, list(seen)


def test_the_module_exports_the_extension():
    for n in TAKES:
        assert getattr(cg, "codegemm_" + n) is getattr(binding._calls, "codegemm_" + n)


@pytest.mark.parametrize("status", [0, -1, -3])
@pytest.mark.parametrize("name", list(TAKES))
def test_forms(calls, name, status):
    seen, result = calls
    result[0] = status
    fast, slow, takes = getattr(cg, "codegemm_" + name), getattr(binding, "_" + name), TAKES[name]
    plain = [GIVEN[t] if t in GIVEN else 12 + k if t in (i32, sz) else Tensor(0x1000 * (k + 1)) for k, t in enumerate(takes)]
    forms = [plain, plain + [77], plain + [0], plain + [2**64 - 16], plain + [None], plain + [3.0], plain + [vp(9)], plain + [-1], plain + [1, 2], plain[:-1], []]
    for k, t in enumerate(takes):
        if t in GIVEN:
            others = [None, 7, CACHE, APPEND, ATTN, cg.Desc.make(1, 512, 512, 8, 1)]
        elif t is vp:
            others = [None, 0, 1, 2**63 + 8, 2**70, -8, True, "x", Tensor(0), Tensor([]), Tensor(RuntimeError("none")), Tensor(KeyboardInterrupt()), Tensor(AttributeError("x"))]
        else:
            others = [0, -1, 2**31 - 1, 2**31, -2**31, 2**40, 2**70, 4.0, None, "n", True]
        forms += [[*plain[:k], o, *plain[k + 1:], *rest] for o in others for rest in ((), (5,))]
    for args in forms:
        assert outcome(fast, seen, *args) == outcome(slow, seen, *args), args
    assert outcome(fast, seen, *plain, 5)[1], "the plain form has to arrive"
    last = slow.__code__.co_varnames[len(takes) - 1]
    for kwargs in ({last: plain[-1]}, {last: plain[-1], "stream": 5}, {last: plain[-1], "stray": 1}):
        assert outcome(fast, seen, *plain[:-1], **kwargs) == outcome(slow, seen, *plain[:-1], **kwargs)


@pytest.mark.parametrize("name", list(TAKES))
def test_what_a_data_ptr_raises_once(calls, name):
    seen, _ = calls

    class Once:
        asked = 0

        def data_ptr(self):
            self.asked += 1
            if self.asked == 1:
                raise KeyboardInterrupt("once")
            return 0x40

    takes = TAKES[name]
    for at in [k for k, t in enumerate(takes) if t is vp]:
        once = Once()
        args = [once if k == at else GIVEN.get(t, 64) for k, t in enumerate(takes)]
        with pytest.raises(KeyboardInterrupt):
            getattr(cg, "codegemm_" + name)(*args, 0)
        assert once.asked == 1 and not seen
