"""What a kernel's launch makes of the library's answers."""
import pytest

from paper_2605_30574_gb300 import decoder as K


@pytest.fixture
def answer(monkeypatch):
    """A library whose functions all give this."""
    def of(rc):
        class Library:
            def __getattr__(self, name):
                return lambda *args: rc
        monkeypatch.setattr(K, "_LIB", Library())
    monkeypatch.setattr(K, "_current_device", lambda: 0)
    monkeypatch.setattr(K, "_raw_stream", lambda device: 0)
    return of


NAMES = ("decoder_page_rows", "decoder_page_copy", "decoder_gemm", "decoder_attention", "decoder_distill", "decoder_page_attention")


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("rc", [1, 700, -1, -2, -700])
def test_an_error_is_raised(answer, name, rc):
    answer(rc)
    with pytest.raises(RuntimeError, match=f"{name} failed with CUDA error {rc}"):
        K._launch(name, 5, 16)


@pytest.mark.parametrize("name", NAMES)
def test_a_launch_that_went_well(answer, name):
    answer(0)
    assert K._launch(name, 5, None) is None


def test_only_an_attention_without_scratch_may_ask_for_some(answer):
    answer(-1)
    assert K._launch("decoder_page_attention", 5, None) is False
    for name in NAMES[:-1]:
        with pytest.raises(RuntimeError, match="error -1"):
            K._launch(name, 5, None)
    answer(-2)
    with pytest.raises(RuntimeError, match="error -2"):
        K._launch("decoder_page_attention", 5, None)
