"""The example of a decoder layer: prompts, then tokens from a captured step."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,batch,longest", [(5, 3, 200), (40, 8, 1500)])
def test_decoder_layer(tokens, batch, longest):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_layer.py")
    spec = importlib.util.spec_from_file_location("decoder_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    assert module.main(tokens, batch, longest) <= 1.0
