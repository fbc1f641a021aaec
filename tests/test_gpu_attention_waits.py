"""Failure detection inside the attention kernels, with no GPU fault.

The warps of a CTA wait for one another with a limit of about two seconds.  The
test hook makes the waits for queries see none (a load that nothing issues) and
give up after about a millisecond: the call must report PTC_ERR_TIMEOUT, with
the copies in flight landed and tensor memory free, so that the calls after it
on the same device are right."""
import time

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_28870_gb300 as ptc
    ptc.lib()


# single tokens, chunks, both; a context cut over many CTAs; requests of few key
# tiles, whose copies are all issued before anything waits; pages without tensor
# copies; the weights by kept scores and by tiles
CASES = {
    "tokens": dict(lens=[(1, 700), (1, 40)], D=128),
    "long token": dict(lens=[(1, 40_000)], Hq=8, Hkv=1, D=128),
    "one key tile": dict(lens=[(40, 40), (3, 3)], D=128),
    "chunks": dict(lens=[(300, 900), (1, 77), (130, 130)], D=128),
    "chunks, 64 columns": dict(lens=[(300, 900), (1, 77)], D=64, dtype="fp16"),
    "long chunk": dict(lens=[(200, 9000)], Hq=8, Hkv=1, D=128),
    "pages of 7": dict(lens=[(100, 300), (1, 900)], D=128, B=7),
}


@pytest.mark.parametrize("with_mass", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_given_up_waits_then_right_results(case, with_mass):
    import torch
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache, check_attention
    c = Cache(**CASES[case])
    mass = torch.zeros(c.Hkv, c.slots, device="cuda") if with_mass else None
    call = lambda **k: ptc.ptc_paged_attention(c.q, *c.table(), c.tok_off, c.kv_len, max(c.new), mass=mass, **k)
    call()  # everything is loaded
    torch.cuda.synchronize()
    L = ptc.lib()
    L.ptc_test_wait_polls(ptc.PTC_TEST_WAIT_ATTENTION + 2000)
    try:
        began = time.perf_counter()
        with pytest.raises(ptc.PtcError) as e:
            call()
        assert e.value.name == "PTC_ERR_TIMEOUT"
        # no wait for a copy or a product that does not come (those have two seconds)
        assert time.perf_counter() - began < 1.0
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        call(status=status)
        with pytest.raises(ptc.PtcError) as e:
            ptc.check_status(status)
        assert e.value.name == "PTC_ERR_TIMEOUT"
    finally:
        L.ptc_test_wait_polls(0)
    for _ in range(2):
        check_attention(c, mass=mass)


def test_other_hooks_leave_the_attention_alone():
    import paper_2609_28870_gb300 as ptc
    from tests.kv_util import Cache, check_attention
    c = Cache([(1, 300), (40, 200)], D=64)
    L = ptc.lib()
    for polls in (300, ptc.PTC_TEST_WAIT_PIECES + 300):
        L.ptc_test_wait_polls(polls)
        try:
            check_attention(c)
        finally:
            L.ptc_test_wait_polls(0)
