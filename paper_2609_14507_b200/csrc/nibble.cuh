// The 4-bit cache format: where every code, scale and zero of a tile lies.
//
// A group of values is held as codes 0..15 with a bf16 scale and zero (value = scale * code + zero).  Groups: the 64 columns
// of one panel of K, all columns of V (per token and KV head).  A block of bt tokens (a multiple of 64) holds, for each KV
// head, bt / 64 tiles of 64 tokens.  A tile is K codes (32 D bytes), K scales and zeros, V codes (32 D), V scales and zeros.
//
// The codes lie in the order in which the lanes of a warp feed them to 16 x 8 tensor-core products as 16-row operands (rows =
// tokens for K, rows = columns of the head for V), so that a lane's 16 bytes are its operands, a warp's 512 bytes are consecutive, and
// no value ever moves between lanes.  With lane = 4 g + t, nibble j = bits 4j..4j+3 of a 32-bit word:
//   K: token 16u + 8h + g, column 64p + 16t + 8w + j  ->  nibble j of word ((((u P + p) 8 + g) 4 + t) 2 + h) 2 + w     (P = D/64)
//   V: column 16d + 8h + g, token 32w + 8i + 2t + e   ->  nibble i + 4e of word ((((d 8 + g) 4 + t) 2 + h) 2 + w
// Masking a word with 0x000f000f leaves nibbles 0 and 4 as the two halves of a register: read as bf16 these bits are the code times
// 2^-133, exactly (a subnormal), and nibbles 1 and 5 in place the code times 2^-129; shifted by three they are as good as fp16.  So codes
// become 16-bit operands with one logical operation per two values, and the powers of two go into the other operand.
// Scales and zeros (scale in the low half of a 32-bit word) are in the rows' order too: token 16u + 8h + g is row 16u + 2g + h.
#pragma once
#include <cstdint>

#include "layout.cuh"

namespace ipkvi {

struct NibbleGeom {
    int32_t n_kv_heads, dim, bt;
    IPKV_HD int32_t panels() const { return dim / 64; }
    IPKV_HD int32_t codes_bytes() const { return 32 * dim; }                                  // of K or V
    IPKV_HD int32_t k_meta_off() const { return codes_bytes(); }
    IPKV_HD int32_t v_off() const { return k_meta_off() + 256 * panels(); }
    IPKV_HD int32_t v_meta_off() const { return v_off() + codes_bytes(); }
    IPKV_HD int32_t tile_bytes() const { return v_meta_off() + 256; }                         // 8960 for 128 columns, 4608 for 64
    IPKV_HD int64_t head_bytes() const { return int64_t(bt / kTileTokens) * tile_bytes(); }
    IPKV_HD int64_t block_bytes() const { return head_bytes() * n_kv_heads; }
    // byte offset of tile `tile` (64 tokens) of a run of consecutive blocks, for one KV head
    IPKV_HD int64_t tile_off(int64_t tile, int32_t head) const {
        const int32_t per = bt / kTileTokens;
        const int64_t blk = tile / per;
        return blk * block_bytes() + int64_t(head) * head_bytes() + (tile - blk * per) * tile_bytes();
    }
};

// Word index inside the K codes of the 8 columns 8c..8c+7 of token t (0..63); nibble j is column 8c + j.
IPKV_HD int32_t nibble_k_word(int32_t panels, int32_t t, int32_t c) {
    const int32_t u = t >> 4, h = (t >> 3) & 1, g = t & 7, p = c >> 3, tt = (c & 7) >> 1, w = c & 1;
    return ((((u * panels + p) * 8 + g) * 4 + tt) * 2 + h) * 2 + w;
}
// Word index inside the V codes of column `col` for the 8 tokens 32w + 8i + 2tt + e; and the nibble of one of them.
IPKV_HD int32_t nibble_v_word(int32_t col, int32_t w, int32_t tt) {
    const int32_t d = col >> 4, h = (col >> 3) & 1, g = col & 7;
    return (((d * 8 + g) * 4 + tt) * 2 + h) * 2 + w;
}
IPKV_HD int32_t nibble_v_of(int32_t t) { return ((t >> 3) & 3) + 4 * (t & 1); }               // w = t >> 5, tt = (t & 7) >> 1
// Row of token t among the scales and zeros.
IPKV_HD int32_t nibble_meta_row(int32_t t) { return (t & 48) + 2 * (t & 7) + ((t >> 3) & 1); }

}  // namespace ipkvi
