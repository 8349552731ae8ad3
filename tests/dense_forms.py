"""Shared by the tests of every form of the dense layers' products, pinned by the switches LUTNN_DENSE_FORM and LUTNN_DENSE_SPLITS."""
# tile sizes by form; those that read their operands as they are lay nothing out
TILES = {"256x256": (256, 256), "128x256": (128, 256), "128x128": (128, 128), "64x128": (64, 128), "64x64": (64, 64), "32x64": (32, 64),
         "64x64 as is": (64, 64), "32x64 as is": (32, 64), "32x32 as is": (32, 32)}
FORMS = {"f32": ("memory", "128x256", "128x128", "64x64 as is", "32x32 as is"),
         "bf16": ("256x256", "128x128", "64x128", "64x64", "32x64", "64x64 as is", "32x64 as is")}
FORMS["f16"] = FORMS["bf16"]
