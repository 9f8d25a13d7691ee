"""The serving entry points from several Python threads."""
import threading
import time

import pytest
import torch

from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu


def test_other_threads_run_while_a_call_waits_for_the_library():
    """One thread asks for a status and waits for the stream in the library, another calls an entry point and waits for the library: a third one goes on."""
    ints = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    tables, lens, refs, one = ints(2, 3) - 1, ints(2), ints(4), ints(1)
    free = lambda: psa.psa_pages_free(tables, lens, refs, one, 16)  # noqa: E731
    free()
    assert psa.psa_last_issued()[0] == psa.OK
    status = []
    asks, calls = threading.Thread(target=lambda: status.append(psa.psa_last_issued()[0])), threading.Thread(target=free)
    torch.cuda._sleep(1_000_000_000)             # about half a second
    begin = last = time.perf_counter()
    asks.start()
    time.sleep(0.05)
    calls.start()
    gap = 0.0
    while calls.is_alive() or asks.is_alive():
        time.sleep(0.002)
        now = time.perf_counter()
        gap, last = max(gap, now - last), now
    asks.join()
    calls.join()
    assert status == [psa.OK] and last - begin > 0.3
    assert gap < 0.15, gap


def test_refusals_still_raise():
    q = torch.zeros(2, 2, 12, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(psa.PsaError) as e:
        psa.psa_prompt_attention(q, q, q, torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    assert e.value.status == psa.ERR_UNSUPPORTED and "psa_prompt_attention" in str(e.value)
