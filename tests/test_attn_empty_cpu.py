"""What stands for no rows and for no keys, and what does not: refusals before anything is enqueued."""
import pytest

from paper_2506_04985_b200 import binding as B
from test_attn_cpu import FAKE, L, gather, prompt  # noqa: F401  (L: the library, a fixture)


@pytest.mark.parametrize("change", [dict(M=0), dict(M=0, K=None), dict(M=0, V=None), dict(M=-1, K=None, V=None), dict(M=-1), dict(K=None, V=None)])
def test_read_back_of_no_rows_has_no_buffers(L, change):  # noqa: F811
    assert gather(L, **change) == B.ERR_BAD_ARG


@pytest.mark.parametrize("change", [dict(Mk=0), dict(Mk=0, K=None), dict(Mk=0, V=None), dict(Mk=-1, K=None, V=None), dict(K=None, V=None),
                                    dict(Mk=0, K=None, V=None, Mq=0), dict(Mk=0, K=None, V=None, ld_k=8), dict(Mk=0, K=None, V=None, Q=None)])
def test_prompt_of_no_keys_has_no_buffers(L, change):  # noqa: F811
    assert prompt(L, **change) == B.ERR_BAD_ARG


def test_what_else_a_call_without_rows_has_to_have(L):  # noqa: F811
    for change, code in ((dict(ws=None), B.ERR_WORKSPACE), (dict(cu=None), B.ERR_BAD_ARG), (dict(first=FAKE + 1), B.ERR_ALIGNMENT)):
        assert gather(L, M=0, K=None, V=None, **change) == code
    for change, code in ((dict(ws=None), B.ERR_WORKSPACE), (dict(hd=80), B.ERR_UNSUPPORTED), (dict(scale=0.0), B.ERR_BAD_ARG)):
        assert prompt(L, Mk=0, K=None, V=None, **change) == code
