"""Tensors that a call of include/ress_pages.h's binding needs and is not given: refused by name before the entry point is called
(CPU only, as tests/test_pages_binding.py)."""
import pytest

from test_pages_binding import _i, _z, pages, traced  # noqa: F401  (fixtures)

Q, K, KP, T = _z(2, 9, 64), _z(1, 9, 64), _z(3, 1, 4, 64), _i(2, 5)
NEEDED = {  # arguments of a call that is complete; the names of those that it needs
    "ress_qk_norm_rope": (dict(q=Q, k=K, pos=_i(9, 1), dims=(64,)), ("pos",)),
    "ress_qk_norm_rope_pages": (dict(q=Q, k=K, v=K, pos=_i(9, 1), slots=_i(9), k_pages=KP, v_pages=KP, dims=(64,)),
                                ("k", "v", "pos", "slots", "k_pages", "v_pages")),
    "ress_qk_norm_rope_bwd": (dict(dq_out=Q, dk_out=K, q=Q, k=K, pos=_i(9, 1), dims=(64,)), ("dq_out", "dk_out", "pos")),
    "ress_page_tables": (dict(lens=_i(2), new_lens=_i(2), tables=T, free_pages=_i(9), n_free=_i(1), page=4, tokens=7),
                         ("lens", "new_lens", "tables", "free_pages", "n_free")),
    "ress_pages_release": (dict(first=_i(2), last=_i(2), tables=T, free_pages=_i(9), n_free=_i(1)),
                           ("first", "last", "tables", "free_pages", "n_free")),
    "ress_paged_attn": (dict(q=Q, k_pages=KP, v_pages=KP, cu_q=_i(3), lens=_i(2), tables=T, window=5),
                        ("q", "k_pages", "v_pages", "cu_q", "lens", "tables")),
}


@pytest.mark.parametrize("name", NEEDED)
def test_missing_tensors_are_refused_by_name(pages, traced, name):  # noqa: F811
    _, calls = traced
    args, needed = NEEDED[name]
    call = getattr(pages, name)
    call(**args)
    assert len(calls) == 1
    for n in needed:
        with pytest.raises(ValueError, match=n.split("_")[0]):
            call(**dict(args, **{n: None}))
    assert len(calls) == 1


def test_gradients_of_one_of_q_and_k(pages, traced):  # noqa: F811
    """Either pair may be left out, its gradient with it."""
    _, calls = traced
    args = NEEDED["ress_qk_norm_rope_bwd"][0]
    pages.ress_qk_norm_rope_bwd(**dict(args, k=None, dk_out=None))
    pages.ress_qk_norm_rope_bwd(**dict(args, q=None, dq_out=None))
    assert len(calls) == 2
