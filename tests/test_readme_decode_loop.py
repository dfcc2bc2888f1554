"""The README's decode loop over the 8-bit cache keeps the order that test_gpu_kv8_layer_order.py checks on the GPU: per layer a write
and then attention over one entry more, and the tables and lengths after the last layer."""
import os


def test_write_then_attend_then_update():
    text = open(os.path.join(os.path.dirname(__file__), os.pardir, "README.md")).read()
    loop = text[text.index("while generating"):]
    loop = loop[:loop.index("```")]
    at = [loop.index(x) for x in ("attended = seq_lens + 1", "for layer", "umim_kv8_write(", "umim_decode_attention_shared_kv8(",
                                  "umim_kv8_append_merge(")]
    assert at == sorted(at)
    attend = loop[at[3]:at[4]]
    assert "block_table, attended" in attend and "seq_lens" not in attend
