"""What the Python entry points of packed prompts and of the paged cache refuse
before anything is launched: types, dimensions, strides, devices, and sizes that
do not belong together."""
import pytest
import torch

from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu

D, HKV, P, PAGES, S, T = 128, 2, 64, 6, 3, 6
BF16, I32, F32 = torch.bfloat16, torch.int32, torch.float32


def _args():
    return dict(q=torch.zeros((1, 4, T, D), dtype=BF16, device="cuda"),
                k=torch.zeros((1, HKV, T, D), dtype=BF16, device="cuda"),
                v=torch.zeros((1, HKV, T, D), dtype=BF16, device="cuda"),
                pages=eb.new_cache_pages(PAGES, HKV, P),
                table=torch.zeros((S, 2), dtype=I32, device="cuda"),
                lengths=torch.full((S,), 2, dtype=I32, device="cuda"),
                cu=torch.tensor([0, 2, 4, T], dtype=I32, device="cuda"))


def _store(a):
    return eb.cache_store(a["k"], a["v"], a["pages"], a["table"], a["lengths"], a["cu"])


def _attn(a):
    return eb.cache_attn(a["q"], a["pages"], a["table"], a["lengths"], a["cu"], out=a.get("out"),
                         workspace=a.get("workspace"), softmax_scale=a.get("scale"))


def _packed(a):
    return eb.packed_prefill_attn(a["q"], a["k"], a["v"], a["cu"], out=a.get("out"),
                                  softmax_scale=a.get("scale"))


def _strided(t):
    """The same values, every second element of a larger tensor."""
    return torch.stack([t, t], -1)[..., 0]


TOKENS = [("not a tensor", lambda t: [0.0], TypeError), ("half", lambda t: t.half(), TypeError),
          ("on the CPU", lambda t: t.cpu(), ValueError), ("strided", _strided, ValueError),
          ("3-d", lambda t: t[0], ValueError),
          ("a batch", lambda t: torch.cat([t, t]), ValueError),
          ("another head_dim", lambda t: t[..., :64].contiguous(), (ValueError, eb.EIError))]
LISTS = [("not a tensor", lambda t: [0], TypeError), ("int64", lambda t: t.long(), TypeError),
         ("on the CPU", lambda t: t.cpu(), ValueError), ("strided", _strided, ValueError),
         ("another dimension", lambda t: t[None], ValueError),
         ("one more", lambda t: torch.cat([t, t[:1]]), ValueError)]
CALLS = [(_store, "k", TOKENS), (_store, "v", TOKENS), (_store, "table", LISTS),
         (_store, "lengths", LISTS), (_store, "cu", LISTS[1:]), (_attn, "q", TOKENS),
         (_attn, "table", LISTS), (_attn, "lengths", LISTS), (_attn, "cu", LISTS[1:]),
         (_packed, "q", TOKENS), (_packed, "k", TOKENS), (_packed, "v", TOKENS),
         (_packed, "cu", LISTS[:-1])]
CASES = [(call, name, what, edit, err) for call, name, edits in CALLS
         for what, edit, err in edits]


@pytest.mark.parametrize("call,name,what,edit,err", CASES,
                         ids=[f"{c[0].__name__[1:]}-{c[1]}-{c[2]}" for c in CASES])
def test_tensors(call, name, what, edit, err):
    a = _args()
    call(a)
    a[name] = edit(a[name])
    with pytest.raises(err):
        call(a)


PAGE_EDITS = [
    ("codes of another type", lambda p: p._replace(k=p.k.float()), TypeError),
    ("two formats", lambda p: p._replace(v=p.v.view(torch.uint8).view(torch.int8)), TypeError),
    ("no tensor", lambda p: p._replace(v_scale=1.0), TypeError),
    ("scales in bf16", lambda p: p._replace(k_scale=p.k_scale.to(BF16)), TypeError),
    ("scales of the CPU", lambda p: p._replace(v_scale=p.v_scale.cpu()), ValueError),
    ("codes of the CPU", lambda p: p._replace(k=p.k.cpu()), ValueError),
    ("strided scales", lambda p: p._replace(k_scale=_strided(p.k_scale)), ValueError),
    ("fewer V pages", lambda p: p._replace(v=p.v[1:]), ValueError),
    ("fewer scales", lambda p: p._replace(v_scale=p.v_scale[1:]), ValueError),
    ("scales of 1 dimension", lambda p: p._replace(k_scale=p.k_scale.view(-1)), ValueError),
    ("two layers", lambda p: eb.new_cache_pages(PAGES, HKV, P, n_layers=2), ValueError),
    ("three dimensions", lambda p: p._replace(k=p.k[0], v=p.v[0]), ValueError),
    ("pages of 32", lambda p: eb.new_cache_pages(PAGES, HKV, 32), eb.EIError),
    ("another KV head", lambda p: eb.new_cache_pages(PAGES, 3, P), ValueError),
    ("another head_dim", lambda p: eb.new_cache_pages(PAGES, HKV, P, 64), ValueError),
]


@pytest.mark.parametrize("call", [_store, _attn])
@pytest.mark.parametrize("what,edit,err", PAGE_EDITS, ids=[e[0] for e in PAGE_EDITS])
def test_pages(call, what, edit, err):
    a = _args()
    a["pages"] = edit(a["pages"])
    with pytest.raises(err):
        call(a)


@pytest.mark.parametrize("call", [_attn, _packed])
def test_output_and_scale(call):
    for out in (torch.empty((1, 4, T + 1, D), dtype=BF16, device="cuda"),
                torch.empty((1, 4, T, D), dtype=BF16),
                _strided(torch.empty((1, 4, T, D), dtype=BF16, device="cuda"))):
        with pytest.raises(ValueError):
            call({**_args(), "out": out})
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(eb.EIError):
            call({**_args(), "scale": scale})


def test_tokens_that_do_not_divide():
    a = _args()
    a["cu"] = None
    _store(a), _attn(a)
    a["lengths"], a["table"] = a["lengths"].repeat(2)[:4], a["table"].repeat(2, 1)[:4]
    for call in (_store, _attn):
        with pytest.raises(ValueError, match="cu_seqlens"):
            call(a)
    a["lengths"], a["table"] = a["lengths"][:0], a["table"][:0]
    for call in (_store, _attn):
        with pytest.raises(ValueError, match="cu_seqlens"):
            call(a)


def test_workspace_of_too_few_bytes():
    a = _args()
    a["table"] = torch.zeros((S, 100), dtype=I32, device="cuda")
    nb = eb.cache_attn_workspace_bytes(4, T, True, S, 100, a["pages"])
    assert nb > 0
    a["workspace"] = torch.empty((nb,), dtype=torch.uint8, device="cuda")
    _attn(a)
    for ws in (a["workspace"][:-1], a["workspace"][16:]):
        a["workspace"] = ws
        with pytest.raises(eb.EIError):
            _attn(a)
    a["workspace"] = torch.empty((nb + 16,), dtype=torch.uint8, device="cuda")[1:]
    with pytest.raises(eb.EIError):      # not aligned
        _attn(a)
    a["workspace"] = torch.empty((nb,), dtype=torch.uint8)
    with pytest.raises(ValueError):
        _attn(a)


def test_copy():
    pages = eb.new_cache_pages(PAGES, HKV, P, n_layers=2)
    one, two = (torch.arange(n, dtype=I32, device="cuda") for n in (1, 2))
    eb.cache_copy(pages, one, one + 1)
    for src, dst, err in ((one, two, ValueError), (one.long(), one, TypeError),
                          (one.cpu(), one, ValueError), (one, one[None], ValueError)):
        with pytest.raises(err):
            eb.cache_copy(pages, src, dst)
    with pytest.raises(ValueError):
        eb.cache_copy(pages._replace(k=pages.k[0]), one, one + 1)
    with pytest.raises(TypeError):
        eb.new_cache_pages(PAGES, HKV, P, dtype=torch.uint8)
