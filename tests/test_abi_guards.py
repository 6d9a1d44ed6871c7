"""Host-side guards, no GPU: sizes at which 32 bits end."""
import pytest

P = 0x10000            # fake, aligned, never dereferenced: every call below is refused before a launch
UNSUPPORTED, WORKSPACE = 3, 5


@pytest.fixture(scope="module")
def ac():
    from paper_2606_07665_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def attention(ac, num_pages, ps, page, token, head):
    c = ac.AcQ4Cache(P, P, P, page, token, head, 64)
    return ac.lib().ac_paged_decode_attn_q4(P, c, P, 33, P, 1, 0.0, 4, None, 0, P, 1, 8, 2, 64, ps, num_pages, 513, None, None, None)


@pytest.mark.parametrize("num_pages,ps,page,token,head", [
    (64, 16, 1 << 31, 64, 32),                        # pages far apart
    (1 << 20, 64, 1 << 12, 1 << 32, 32),              # slot-major: 64 slots of a million pages' 4096 bytes, 2^38 bytes
    (2, 256, 1 << 10, 1 << 29, 32),                   # a token stride that no page stride explains
    (2, 256, 1 << 62, 1 << 62, 32),                   # products past 64 bits
    (1 << 30, 256, 1 << 40, 1 << 40, 32),
    (2, 32, 64, (1 << 36) // 16 + 16, 32)])           # just past the border
def test_code_pools_of_more_than_36_bits_are_refused(ac, num_pages, ps, page, token, head):
    assert attention(ac, num_pages, ps, page, token, head) == UNSUPPORTED


@pytest.mark.parametrize("num_pages,ps,page,token,head", [
    (1, 16, 1 << 60, 64, 32),                         # one page: its stride is never used
    (2, 16, 1 << 35, 1 << 60, 32),                    # one granule per page: the token stride stays in 64 bits
    (1 << 18, 64, 64, 64 << 18, 32),                  # slot-major, 2^30 bytes
    (2, 32, 64, (1 << 36) // 16 - 16, 32)])           # just within
def test_code_pools_within_36_bits_pass_that_guard(ac, num_pages, ps, page, token, head):
    # what stops them here is the workspace that four splits want, looked at after the pools
    assert attention(ac, num_pages, ps, page, token, head) == WORKSPACE


@pytest.mark.parametrize("Hkv", [1, 8])
def test_plans_for_two_billion_tokens(ac, Hkv):
    # the split count of a context at the end of 32 bits is that of one a little shorter, and known lengths of the whole
    # context give the plan that unknown ones give
    near, end = 2**30 - 64, 2**31 - 1
    want = ac.ac_decode_plan_q4(None, 1, 8, Hkv, 64, 16, near, 148)[0]
    assert want > 1
    assert ac.ac_decode_plan_q4(None, 1, 8, Hkv, 64, 16, end, 148)[0] == want
    assert ac.ac_decode_plan_q4([end], 1, 8, Hkv, 64, 16, end, 148)[0] == want
    want = ac.ac_decode_plan(1, 8, Hkv, 64, 16, end, 148)
    assert want[0] == ac.ac_decode_plan(1, 8, Hkv, 64, 16, near, 148)[0]
    assert ac.ac_decode_plan_for_lengths([end], 8, Hkv, 64, 16, end, 148) == want


def test_trim_refusals(ac):
    def trim(table=P, mp=8, lens=P, refs=P, rows=4, ps=16, pages=64):
        return ac.lib().ac_cache_trim(table, mp, lens, refs, rows, ps, pages, None, None)

    assert trim(table=None) == trim(lens=None) == trim(refs=None) == 1
    assert trim(mp=0) == trim(rows=0) == trim(ps=0) == trim(pages=0) == trim(pages=-5) == 2
    assert trim(pages=2**30 + 1) == UNSUPPORTED


@pytest.mark.parametrize("d,group", [(128, 48), (128, 100), (64, 128), (64, 0), (128, -64), (128, 16), (64, 65)])
def test_an_empty_cache_has_the_group_that_was_asked_for_or_none(d, group):
    from paper_2606_07665_b200 import runner
    with pytest.raises(ValueError, match="group"):
        runner.Q4Cache.empty(4, 16, 2, d, group=group)


def test_unknown_layouts_are_refused():
    from paper_2606_07665_b200 import runner
    with pytest.raises(ValueError, match="layout"):
        runner.Q4Cache.empty(4, 16, 2, 64, layout="headmajor")
