"""What the feed-forward block's command says of a step that went wrong."""
import pytest
import torch

from paper_2010_14298_gb300 import ffn, fqt

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


def test_the_command_names_the_condition():
    """An infinite learning rate leaves weights that are not finite, which the next
    step's quantizers record."""
    with pytest.raises(SystemExit, match=fqt.status_string(4)):
        ffn.main(["--tokens", "64", "--width", "64", "--hidden", "128", "--steps", "3", "--lr",
                  "inf"])
