"""GPU: the example that runs the price loop and the paged cache together."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_a_job_goes_on_in_a_smaller_budget():
    import elastic_inference as example
    print("[gpu-case] elastic inference", flush=True)
    r = example.main(steps=5)
    wide, narrow = r["batches"]
    assert r["status"] == 0 and narrow < wide and len(r["lengths"]) == narrow
    assert r["pages"] == (wide * example.PAGES_A_SEQUENCE, narrow * example.PAGES_A_SEQUENCE) and r["highest"] < r["pages"][1]
    assert r["freed"] == (wide - narrow) * example.PAGES_A_SEQUENCE
    assert r["lengths"][:4] == [example.PROMPT - 7 * i + 10 for i in range(min(4, narrow))]
    # weights and output rounded to fp16 (2^-11 of the largest value each), the rest far below
    assert max(r["errors"]) <= 3 * 2.0 ** -11
