"""The mixture-of-experts command refuses what it cannot do before anything is made on a GPU."""
import pytest

from paper_1705_01598_amd import experts as E


@pytest.mark.parametrize("arguments", [["--bits", "4"], ["--answer", "--bits", "32"], ["--bits", "32"], ["--answer", "--bits", "16", "--dtype", "f32"],
                                       ["--bits", "4", "--dtype", "f16"]])
def test_bits_that_are_not_the_types(arguments, capsys):
    with pytest.raises(SystemExit) as e:
        E._bench(arguments)
    assert e.value.code == 2 and "--bits: 4 with --answer, or those of the type" in capsys.readouterr().err
