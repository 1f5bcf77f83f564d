"""Windows of the 4-bit cache up to the type's end, with rows that stand before a request's first token: the arithmetic of the kernels' own header, run on
the host, against Python's integers.  No GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2109_10060_b200", "csrc")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("window") / "cache_window")
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", os.path.join(ROOT, "include"),
                    "-I", CSRC, os.path.join(ROOT, "tests", "cache_window.cu"), "-o", out], check=True)
    return out


def test_every_window_and_every_token(program):
    ends = (0, 1, 2, 3, 15, 16, 17, 1000, 2 ** 24, 2 ** 29, 2 ** 30 - 16, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 1, 2 ** 31 - 2 ** 24, 2 ** 31 - 3, 2 ** 31 - 2, 2 ** 31 - 1)
    asked = []
    for pages, page in ((1, 16), (5, 48), (2 ** 20 - 1, 1024), (2 ** 26 - 1, 16)):
        room = pages * page
        for window in sorted({*ends, *(room + o for o in (-2, -1, 0, 1))}):
            for me in (-2 ** 24, -2 ** 23, -4, -3, -2, -1, 0, 1, 2, 15, 16, 17, room // 2, room - 2, room - 1):
                if me < room:
                    asked.append((pages, page, window, me))
    out = subprocess.run([program], input="".join("%d %d %d %d\n" % a for a in asked), check=True, capture_output=True, text=True).stdout.split()
    got = list(zip(map(int, out[0::2]), map(int, out[1::2])))
    assert len(got) == len(asked)
    for (pages, page, window, me), (held, first) in zip(asked, got):
        assert 0 <= held < 2 ** 30
        assert first == (max(0, me - window + 1) if window else 0), (pages, page, window, me)
        # differences that the kernels' masks make
        assert -2 ** 31 <= me - held and -2 ** 31 <= pages * page - 1 - held


@pytest.mark.parametrize("source", ["dsn_cache_attention.cu", "dsn_cache_attention_rows.cu"])
def test_a_window_reaches_the_kernels_through_that_arithmetic_alone(source):
    """No sum `... - window + 1` of their own that starts from a row before the first token."""
    text = open(os.path.join(CSRC, source)).read()
    assert "dsn_cache_first_seen" in text and "- window + 1)" not in text
    assert "p.window = dsn_cache_window(" in open(os.path.join(CSRC, "dsn_api.cu")).read()
